"""The operators that mix tokens where calls are at their edges: no tokens, values that are infinite or not a number, positions far out."""
import pytest
import torch

import paper_1804_10727_amd as idf
from test_gpu_tokens import DEV, TYPES, normal

pytestmark = pytest.mark.gpu


# ---- calls without tokens ----

@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dk", [64, 128, 256])
def test_decay_without_tokens_hands_states_on(dtype, in_place, dk, monkeypatch):
    """No stream brings anything, in a call whose bound on the tokens of a segment is that of every other call."""
    from paper_1804_10727_amd import tokens
    g = torch.Generator().manual_seed(40)
    state = torch.randn(3, 2, dk, 64, generator=g).to(DEV)
    q, v = torch.empty(0, 2, dk, dtype=dtype, device=DEV), torch.empty(0, 2, 64, dtype=dtype, device=DEV)
    offsets, log_decay = torch.zeros(4, dtype=torch.int64, device=DEV), torch.tensor([-0.5, -0.1], device=DEV)
    for by_ctypes in (False, True):
        if by_ctypes:
            monkeypatch.setattr(tokens, "_direct", lambda *a: None)
        for max_tokens in (1, 128, 1024, 4096):
            into = state.clone() if in_place else torch.full_like(state, 7.0)
            out = idf.decay_attend(q, q, v, log_decay, into if in_place else state, into, offsets=offsets, max_tokens=max_tokens)
            assert out.shape == (0, 2, 64) and torch.equal(into, state)
            idf.decay_attend(q, q, v, log_decay, None, into, offsets=offsets, max_tokens=max_tokens)
            assert torch.equal(into, torch.zeros_like(state))           # (no states: zeros are handed on)


# ---- values that are infinite or not a number ----

@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 5, 20, 70, 600])
def test_decay_that_is_not_a_number(dtype, n):
    """One head's decay is NaN: all that this head gives is, token by token, in chunks and in parts; the other head's is as without it."""
    g = torch.Generator().manual_seed(41)
    q, k, v = (normal(g, n, 2, 64, dtype=dtype).to(DEV) for _ in range(3))
    state = torch.randn(1, 2, 64, 64, generator=g).to(DEV)
    got = []
    for first in (-0.1, float("nan")):
        end = torch.empty_like(state)
        got.append((idf.decay_attend(q, k, v, torch.tensor([first, -0.2], device=DEV), state, end), end))
    (want, want_end), (out, end) = got
    assert torch.isfinite(want).all() and torch.isnan(out[:, 0]).all() and torch.isnan(end[:, 0]).all()
    assert torch.equal(out[:, 1], want[:, 1]) and torch.equal(end[:, 1], want_end[:, 1])
