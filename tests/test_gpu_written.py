"""What the operators write into tensors of the caller's counts as a change in place, by either way into the library: a backward pass that would start from what
they held before is refused by torch, and not answered from what they hold now."""
import pytest
import torch

import paper_1804_10727_amd as idf
from paper_1804_10727_amd import tokens

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def calls():
    """(name, call, tensors that it writes, tensors that it only reads)"""
    def t(*shape):
        return torch.randn(*shape, device=DEV)
    n, f = 24, idf.rotary_frequencies(64, device=DEV)[0]
    at, x, gates, q, k, v, ring = torch.arange(n, device=DEV), t(n, 64), t(n, 64), t(n, 2, 64), t(n, 1, 64), t(n, 1, 64), idf.nibble_ring(1, 64, 1, 64, DEV)
    rings, out, state, to = [t(1, 64, 1, 64) for _ in range(2)], t(n, 2, 64), t(1, 1, 64, 64), t(1, 1, 64, 64)
    codes, scales = idf.quantize_rows(x)
    y, s0, s1, marks = t(n, 64), t(1, 64), t(1, 64), torch.empty(2 * 64 + 64, device=DEV)
    w, ws, decay = codes[:16].contiguous(), scales[:16].contiguous(), -torch.ones(1, device=DEV)
    qo, ko, z = torch.empty_like(q), torch.empty_like(k), t(n, 16)
    return [("norm_rotate", lambda f_: f_(q, k, at, f, "half", 1.0, None, None, 1e-6, qo, ko), [qo, ko], [q, k, at, f]),
            ("window_attend", lambda f_: f_(q, k, v, *rings, None, 9, 0, None, None, None, None, out), [out, *rings], [q, k, v]),
            ("decay_attend", lambda f_: f_(q, k, v, decay, state, to, None, None, None, None, None, out), [out, to], [q, k, v, state]),
            ("quantize_rows", lambda f_: f_(x, codes, scales), [codes, scales], [x]),
            ("project_rows", lambda f_: f_(x, w, ws, None, None, None, z), [z], [x, w, ws]),
            ("nibble_append", lambda f_: f_(k, v, ring, None, 0, None, "half", 1.0, None, 1e-6, None, None, None), list(ring), [k, v]),
            ("nibble_attend", lambda f_: f_(q, ring, None, 9, 0, None, None, None, None, out), [out], [q, *ring]),
            ("gate_scan", lambda f_: f_(x, gates, s0, s1, None, None, None, None, y, marks), [y, s1, marks], [x, gates, s0])]


SHORT = {"norm_rotate": lambda q, k, at, f, layout, amp, qw, kw, eps, qo, ko: idf.norm_rotate(q, k, at, f, q_out=qo, k_out=ko),
         "window_attend": lambda q, k, v, kr, vr, st, w, s, sc, o, m, ids, out: idf.window_attend(q, k, v, kr, vr, window=w, out=out),
         "decay_attend": lambda q, k, v, d, s, to, sc, o, m, n, ids, out: idf.decay_attend(q, k, v, d, s, to, out=out), "quantize_rows": lambda x, c, s: idf.quantize_rows(x, c, s),
         "project_rows": lambda x, w, ws, b, xs, dt, out: idf.project_rows(x, w, ws, out=out), "nibble_append": lambda k, v, ring, *rest: idf.nibble_append(k, v, ring),
         "nibble_attend": lambda q, ring, st, w, s, sc, o, m, ids, out: idf.nibble_attend(q, ring, window=w, out=out),
         "gate_scan": lambda x, g, s, to, o, m, n, ids, out, marks: idf.gate_scan(x, g, s, to, out=out, marks=marks)}


@pytest.mark.parametrize("way", ["short", "long"])
def test_versions(way):
    for name, call, writes, reads in calls():
        before = [[t._version for t in ts] for ts in (writes, reads)]
        call(SHORT[name] if way == "short" else getattr(tokens, "_" + name))
        assert all(t._version > v for t, v in zip(writes, before[0])) and [t._version for t in reads] == before[1], name


def test_a_saved_tensor_that_is_written_over():
    x, gates = torch.randn(40, 64, device=DEV), torch.randn(40, 64, device=DEV).requires_grad_()
    out, _ = idf.gate_scan_recorded(x, gates)
    w, ws = idf.quantize_rows(torch.randn(64, 64, device=DEV))
    with torch.no_grad():
        idf.project_rows(torch.randn(40, 64, device=DEV), w, ws, out=x)
    with pytest.raises(RuntimeError, match="modified"):
        out.sum().backward()


def test_under_inference_mode():
    with torch.inference_mode():
        for name, call, *_ in calls():
            call(SHORT[name])
            call(getattr(tokens, "_" + name))
    torch.cuda.synchronize()
