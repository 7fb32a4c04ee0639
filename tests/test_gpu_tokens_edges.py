"""The operators that mix tokens where calls are at their edges: no tokens, values that are infinite or not a number, positions far out."""
import numpy as np
import pytest
import torch

import paper_1804_10727_amd as idf
from oracle import tokens as oracle
from test_gpu_tokens import DEV, TYPES, W, decay_case, f64, half_step, normal, rounded, within

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


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("dk", [64, 96, 128])
@pytest.mark.parametrize("n,at", [(1, 0), (4, 1), (40, 0), (40, 33), (40, 39), (600, 7), (600, 130), (600, 599)])
def test_decay_infinite_keys_and_values_stay_in_the_state(dtype, dk, n, at):
    """S gains k^T v: infinite of its sign where one of the two is infinite and the other is not zero, and stays so; the rest is as without it."""
    g = torch.Generator().manual_seed(42)
    q, k, v = (normal(g, n, 1, d, dtype=dtype) for d in (dk, dk, 64))
    log_decay = torch.tensor([-0.02], device=DEV)

    def end(k, v):
        s = torch.randn(1, 1, dk, 64, generator=torch.Generator().manual_seed(43)).to(DEV)
        idf.decay_attend(q.to(DEV), k.to(DEV), v.to(DEV), log_decay, s, s)
        return s[0, 0].cpu()
    want = end(k, v)
    size = float((k.double().abs().amax() * v.double().abs().amax()) * min(n, 60) + 5)
    for row, col, bad in ((None, 3, float("inf")), (None, 60, -float("inf")), (5, None, float("inf")), (dk - 1, None, -float("inf"))):
        kk, vv = k.clone(), v.clone()
        if row is None:
            vv[at, 0, col] = bad
            gained = torch.sign(k[at, 0].float())[:, None] * bad * torch.ones(1, 64)
            hit = torch.zeros(dk, 64, dtype=torch.bool)
            hit[:, col] = True
        else:
            kk[at, 0, row] = bad
            gained = torch.ones(dk, 1) * bad * torch.sign(v[at, 0].float())[None, :]
            hit = torch.zeros(dk, 64, dtype=torch.bool)
            hit[row] = True
        got = end(kk, vv)
        assert torch.equal(got[hit], gained[hit]), (row, col)
        # (the rest by another way in one chunk: float32 sums of 2 n terms in another order)
        assert torch.allclose(got[~hit], want[~hit], rtol=0, atol=4 * (n + 16) * W * size), (row, col)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("dk", [40, 64, 96])
@pytest.mark.parametrize("n,at", [(1, 0), (20, 3), (600, 130)])
def test_decay_infinite_keys_and_values_in_outputs(dtype, dk, n, at):
    """Of queries, keys and values that are all positive an infinite one gives infinity, from its token on, and nothing but that."""
    g = torch.Generator().manual_seed(46)
    q, k, v = (normal(g, n, 1, d, dtype=dtype).abs() + 0.1 for d in (dk, dk, 64))
    log_decay = torch.tensor([-0.02], device=DEV)
    for column, bad in ((7, "value"), (slice(None), "key")):
        kk, vv = k.clone(), v.clone()
        (vv if bad == "value" else kk)[at, 0, 7] = float("inf")
        out = idf.decay_attend(q.to(DEV), kk.to(DEV), vv.to(DEV), log_decay)[:, 0]
        hit = torch.zeros(n, 64, dtype=torch.bool, device=DEV)
        hit[at:, column] = True
        assert torch.all(out[hit] == float("inf")) and torch.isfinite(out[~hit]).all(), bad


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,r", [(64, 8), (64, 24), (64, 4), (80, 20), (18, 6)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_values_behind_the_rotated_ones_stay_by_themselves(dtype, layout, d, r, bad):
    """What is not turned is copied: an infinite value there makes nothing else infinite, nor its neighbour not a number."""
    g = torch.Generator().manual_seed(44)
    x = normal(g, 3, 2, d, dtype=dtype)
    positions, f = torch.tensor([0, 5, 1000], device=DEV), torch.linspace(0.1, 1, r // 2, dtype=torch.float64, device=DEV)
    want, _ = idf.norm_rotate(x.to(DEV), x.to(DEV), positions, f, layout=layout)
    for c in range(r, d):
        y = x.clone()
        y[:, :, c] = bad
        got, _ = idf.norm_rotate(y.to(DEV), y.to(DEV), positions, f, layout=layout)
        w = want.clone()
        w[:, :, c] = bad
        assert torch.equal(torch.nan_to_num(got.float(), nan=12345.0), torch.nan_to_num(w.float(), nan=12345.0)), c


# ---- long streams of slow decays ----

def relative(state, start, log_decay, n):
    """Mean over each head's values of the relative error of what n tokens without keys have left."""
    want = start.double() * torch.exp(log_decay.double() * n)[None, :, None, None]
    return ((state.double() - want) / want).mean(dim=(0, 2, 3)).abs().cpu().numpy()


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_decay_rounding_of_a_factor_does_not_add_up(dtype):
    """A state that nothing is added to, token by token and by parts: float32 roundings of the state, in either direction, cancel over its
    many values; a factor that is off by half a step of float32 would be off in the same direction for all of them.

    Each of n products rounds by at most W.  A slow decay leaves a value nearly where it is, so that its roundings can all be alike, but not those of
    another value: errors of up to n W, independent from value to value, evenly spread (a root of 3 less), leave a mean over m values of at most
    6 n W / sqrt(3 m)."""
    log_decay = -torch.tensor([5e-4, 3.3e-4, 1e-4, 2.7e-5, 1e-6, 4e-3], device=DEV)
    h = len(log_decay)
    g = torch.Generator().manual_seed(45)
    for n, dk, steps in ((4000, 256, 4000), (65536, 64, 65536 // 128 + 4)):        # tokens; parts of 128 tokens, and the last one's chunks
        start = (1 + torch.rand(1, h, dk, 64, generator=g)).to(DEV)
        q, k, v = (torch.zeros(n, h, d, dtype=dtype, device=DEV) for d in (dk, dk, 64))
        end = torch.empty_like(start)
        idf.decay_attend(q, k, v, log_decay, start, end)
        keep = (log_decay * n > -60).cpu().numpy()
        off = relative(end, start, log_decay, n)
        # (the exponent of a part is formed from a float32 logarithm: n |log_decay| W)
        bound = 6 * steps * W / np.sqrt(3 * dk * 64) + n * log_decay.abs().cpu().numpy() * W
        assert np.all(off[keep] <= bound[keep]), (n, off / bound)


# ---- many rows ----

def test_decay_more_query_rows_than_a_launch_axis():
    """9 000 tokens of 1 024 query heads on one: each head as by itself."""
    g = torch.Generator(DEV).manual_seed(47)
    q, k, v = (torch.randn(9000, h, 8, generator=g, device=DEV).bfloat16() for h in (1024, 1, 1))
    log_decay = torch.tensor([-0.01], device=DEV)
    out = idf.decay_attend(q, k, v, log_decay)
    for h in (0, 511, 1023):
        assert torch.equal(out[:, h:h + 1], idf.decay_attend(q[:, h:h + 1].contiguous(), k, v, log_decay))


def test_a_push_of_the_mixer_without_rows():
    from paper_1804_10727_amd.mixing import TokenMixer
    g = torch.Generator().manual_seed(48)
    a, b = (TokenMixer(32, 3, heads=2, kv_heads=1, dim=32, window=8) for _ in range(2))
    for counts in ((2, 0, 1), (0, 0, 0), (1, 30, 2)):
        x = torch.randn(sum(counts), 32, generator=g).to(DEV)
        y = a.push(x, counts)
        assert y.shape == x.shape
        if sum(counts):
            assert torch.equal(y, b.push(x, counts))
    assert a.starts.tolist() == [3, 30, 3] and torch.equal(a.state, b.state)


# ---- gradients ----

def test_tensors_that_require_gradients_are_refused():
    """There is no backward pass: nothing is read, written or lost silently; without recording they are tensors as any other."""
    q, k, v = (torch.randn(4, h, 64, device=DEV) for h in (2, 1, 1))
    f, _ = idf.rotary_frequencies(64, device=DEV)
    rings = [torch.zeros(1, 8, 1, 64, device=DEV) for _ in range(2)]
    p, w, state, into = torch.arange(4, device=DEV), torch.ones(64, device=DEV), torch.zeros(1, 1, 64, 64, device=DEV), torch.empty(4, 2, 64, device=DEV)
    log_decay, start = torch.tensor([-0.1], device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    calls = ((idf.norm_rotate, (q, k, p, f), dict(q_weight=w, k_weight=w.clone(), q_out=into, k_out=torch.empty_like(k))),
             (idf.window_attend, (q, k, v, *rings, start), dict(window=8, out=into)),
             (idf.decay_attend, (q, k, v, log_decay, state, state.clone()), dict(out=into)))
    for call, args, kw in calls:
        call(*args, **kw)
        for t in [*args, *kw.values()]:
            if not torch.is_tensor(t) or not t.is_floating_point():
                continue
            t.requires_grad_(True)
            before = [x.detach().clone() for x in [*args, *kw.values()] if torch.is_tensor(x)]
            with pytest.raises(ValueError, match="gradients"):
                call(*args, **kw)
            assert all(torch.equal(a, b) for a, b in zip(before, [x for x in [*args, *kw.values()] if torch.is_tensor(x)]))
            with torch.no_grad():
                call(*args, **kw)
            t.requires_grad_(False)


# ---- positions far out, offsets that lie, long keys ----

def turns(p, f):
    """Cosine and sine of the exact product of a whole number and a float64 one."""
    from decimal import Decimal, getcontext
    getcontext().prec = 90
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798")
    angle = float((Decimal(p) * Decimal(f)) % (2 * pi))
    return np.cos(angle), np.sin(angle)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_at_positions_beyond_32_bits(dtype, layout):
    """Angles are float64: the product with the frequency, the number of quarter turns in one radian and the product with that are rounded once each,
    2^-53 of the angle.  The rest, taken to a quarter turn, is float32 as anywhere (test_norm_rotate)."""
    g = torch.Generator().manual_seed(49)
    positions = [0, 3, 1 << 24, (1 << 31) - 1, (1 << 31) + 7, (1 << 34) + 12345, (1 << 40) + 99, -(1 << 35) - 1]
    d = 64
    f, amplitude = idf.rotary_frequencies(d, scaling="parts", factor=8.0)
    x = normal(g, len(positions), 2, d, dtype=dtype)
    got, _ = idf.norm_rotate(x.to(DEV), x.to(DEV), torch.tensor(positions, device=DEV), f.to(DEV), layout=layout, amplitude=amplitude)
    want, bound = f64(x).copy(), np.zeros(x.shape)
    for i in range(d // 2):
        a, b = (i, i + d // 2) if layout == "half" else (2 * i, 2 * i + 1)
        for t, p in enumerate(positions):
            c, s = (amplitude * y for y in turns(p, f[i].item()))
            u, v = f64(x)[t, :, a], f64(x)[t, :, b]
            want[t, :, a], want[t, :, b] = u * c - v * s, v * c + u * s
            size = amplitude * (np.abs(u) + np.abs(v))
            bound[t, :, a] = bound[t, :, b] = size * (3 * 2.0 ** -53 * abs(p) * f[i].item() + 32 * W)
    within(got, want, half_step(dtype) * np.abs(want) + bound)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("m", [4, 200])
def test_window_offsets_that_lie_cut_segments_where_they_can(dtype, m):
    """Ends behind the next beginning are cut to the longest segment, ends ahead of their beginning leave nothing, and all to the tokens there are."""
    g = torch.Generator().manual_seed(50)
    n = 3 * m
    q, k, v = (normal(g, n, h, 64, dtype=dtype) for h in (2, 1, 1))
    out = torch.full((n, 2, 64), 9.0, dtype=dtype, device=DEV)
    idf.window_attend(*(x.to(DEV) for x in (q, k, v)), window=1000, offsets=torch.tensor([-5, m, 2 * m + 5, 2 * m, 1 << 40], device=DEV), max_tokens=m, out=out)
    for rows in (slice(0, m), slice(m, 2 * m), slice(2 * m, n)):
        want, size, score = oracle.Attention(1000, 0, 1 / 8).push(*(f64(x[rows]) for x in (q, k, v)))
        within(out[rows], want, half_step(dtype) * np.abs(want) + (rounded(dtype) + 4 * 72 * W * score[..., None] + 2 * (m + 16) * W) * size, rows)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(256, 64), (136, 40)])
def test_decay_long_segments_of_long_keys(dtype, dk, dv):
    decay_case(dtype, 2, 1, dk, dv, (1500, 3, 0, 129), seed=dk)


@pytest.mark.parametrize("dk", [4, 36, 68, 124])
@pytest.mark.parametrize("n,at", [(20, 3), (300, 130)])
def test_decay_infinite_values_with_keys_that_end_inside_a_fragment(dk, n, at):
    """Float32 keys of 4 mod 8 values: what fills the last fragment takes no part."""
    g = torch.Generator().manual_seed(51)
    q, k, v = (normal(g, n, 1, d, dtype=torch.float32).abs() + 0.1 for d in (dk, dk, 64))
    v[at, 0, 7] = float("inf")
    end = torch.empty(1, 1, dk, 64, device=DEV)
    out = idf.decay_attend(q.to(DEV), k.to(DEV), v.to(DEV), torch.tensor([-0.02], device=DEV), None, end)[:, 0]
    hit = torch.zeros(n, 64, dtype=torch.bool, device=DEV)
    hit[at:, 7] = True
    assert torch.all(out[hit] == float("inf")) and torch.isfinite(out[~hit]).all()
    assert torch.all(end[..., 7] == float("inf")) and torch.isfinite(end[..., :7]).all() and torch.isfinite(end[..., 8:]).all()
@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n,calls", [(16, 4000), (32, 3000), (77, 1500)])
def test_decay_rounding_of_a_factor_does_not_add_up_over_calls(dtype, n, calls):
    """The same where a stream brings a few tokens at a time: bounds as above, of the chunks that the calls have; the exponent of a chunk is formed
    from a float32 logarithm in units of log 2, which is rounded twice."""
    log_decay = -torch.tensor([5e-4, 3.3e-4, 1e-4, 2.7e-5, 1e-6], device=DEV)
    h = len(log_decay)
    g = torch.Generator().manual_seed(52)
    start = (1 + torch.rand(4, h, 64, 64, generator=g)).to(DEV)
    state = start.clone()
    q = torch.zeros(4 * n, h, 64, dtype=dtype, device=DEV)
    out = torch.empty_like(q)
    for _ in range(calls):
        idf.decay_attend(q, q, q, log_decay, state, state, out=out)
    off = relative(state, start, log_decay, n * calls)
    bound = 6 * calls * -(-n // 32) * W / np.sqrt(3 * 4 * 64 * 64) + 2 * n * calls * log_decay.abs().cpu().numpy() * W
    assert np.all(off <= bound), off / bound


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("lengths", [(1, 0, 1), (3, 1, 2), (20, 0, 7), (150, 0, 200)])
def test_bounds_beyond_the_tokens_change_nothing(dtype, lengths):
    g = torch.Generator().manual_seed(53)
    n = sum(lengths)
    q, k, v = (normal(g, n, h, 64, dtype=dtype).to(DEV) for h in (4, 1, 1))
    offsets, starts = torch.tensor((0,) + lengths).cumsum(0).to(DEV), torch.tensor([50, 3, 1000], device=DEV)
    rings = [normal(g, 3, 250, 1, 64, dtype=dtype).to(DEV) for _ in range(2)]
    state, log_decay = torch.randn(3, 1, 64, 64, generator=g).to(DEV), torch.tensor([-0.1], device=DEV)
    want = None
    for max_tokens in (n, n + 1, 4096, 1 << 24):
        r, s = [x.clone() for x in rings], state.clone()
        got = [idf.window_attend(q, k, v, *r, starts, window=40, sinks=2, offsets=offsets, max_tokens=max_tokens), *r,
               idf.decay_attend(q, k, v, log_decay, s, s, offsets=offsets, max_tokens=max_tokens), s]
        want = want or got
        assert all(torch.equal(a, b) for a, b in zip(got, want)), max_tokens
