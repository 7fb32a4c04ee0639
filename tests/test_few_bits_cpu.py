"""What the layers in few bits and the gated recurrence refuse, and pins of their oracle: host code, no GPU needed."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_1804_10727_amd as idf
from oracle import few_bits as oracle
from paper_1804_10727_amd import tokens

BUF = C.create_string_buffer(1 << 16)
AT = (C.addressof(BUF) + 255) // 256 * 256         # never read: every call below ends before anything is enqueued
NAN, INF = float("nan"), float("inf")


def rows(stride=64, base=AT):
    return tokens._Rows(base, stride)


def toks(stride=128, head=64, base=AT):
    return tokens._Tokens(base, stride, head)


def ring(**kw):
    return tokens._NibbleRing(*(kw.get(n, AT) for n in ("k_codes", "k_scales", "v_codes", "v_scales")))


def change(a, kw):
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def quantize_args(**kw):
    return change(tokens._Quantize(0, 64, 4, rows(), AT, AT), kw)


def project_args(**kw):
    return change(tokens._Project(0, 0, 64, 32, 4, rows(), rows(), None, AT, AT, None, AT, 1 << 16), kw)


def append_args(**kw):
    return change(tokens._NibbleAppend(0, 2, 64, 32, 0, 4, 4, 1, 1, 16, 2, 1.0, 1e-6, toks(), toks(), ring(), AT, None, None, None, None), kw)


def attend_args(**kw):
    return change(tokens._NibbleAttend(0, 4, 2, 64, 4, 4, 1, 1, 16, 8, 2, 0.125, toks(256), toks(256), ring(), None, None, None, None, 0), kw)


def values_args(**kw):
    return change(tokens._NibbleValues(0, 2, 64, 1, 16, ring(), AT, AT), kw)


def gate_args(**kw):
    return change(tokens._GateScan(0, 64, 4, 4, 1, 1, rows(), rows(), rows(), None, None, None, None, None, None, 0), kw)


def back_args(**kw):
    return change(tokens._GateScanBackward(0, 64, 4, 4, 1, 1, rows(), rows(), rows(), rows(), rows(), None, None, AT, None, None, None, 0), kw)


def refused(fn, a, want):
    assert getattr(idf.load_library(), fn)(C.byref(a) if a is not None else None, None) == want and idf.load_library().idf_last_error()


@pytest.mark.parametrize("kw,want", [
    (dict(precision=2), -5), (dict(cols=0), -5), (dict(cols=65537), -5), (dict(n_rows=-1), -1), (dict(n_rows=1 << 24), -1), (dict(x=rows(base=None)), -1), (dict(x=rows(base=AT + 2)), -1),
    (dict(x=rows(-64)), -5), (dict(x=rows((1 << 25) + 1)), -5), (dict(codes=None), -1), (dict(scales=None), -1), (dict(codes=AT + 8), -5)])
def test_quantize_refuses(kw, want):
    refused("idf_quantize_rows", quantize_args(**kw), want)


@pytest.mark.parametrize("kw,want", [
    (dict(precision=3), -5), (dict(out_precision=2), -5), (dict(cols=0), -5), (dict(cols=1 << 17), -5), (dict(precision=2, cols=40), -5), (dict(n_out=0), -5), (dict(n_out=1 << 25), -5),
    (dict(n_rows=-1), -1), (dict(x=rows(base=None)), -1), (dict(out=rows(base=None)), -1), (dict(out=rows(31)), -1), (dict(out=rows(base=AT + 1)), -1), (dict(weights=None), -1),
    (dict(weight_scales=None), -1), (dict(weights=AT + 4), -5), (dict(precision=2), -1), (dict(precision=2, x_scales=AT, x=rows(72)), -5), (dict(precision=2, x_scales=AT, x=rows(base=AT + 8)), -5),
    (dict(workspace=None), -2), (dict(workspace_bytes=4 * 64 + 15), -2), (dict(workspace=AT + 16), -1)])
def test_project_refuses(kw, want):
    refused("idf_project_rows", project_args(**kw), want)


PACKING = [(dict(precision=2), -5), (dict(n_tokens=-4), -1), (dict(max_tokens=-1), -1), (dict(n_segments=-1), -1), (dict(n_segments=2), -1), (dict(max_tokens=3), -1),
           (dict(n_streams=0), -1), (dict(n_segments=70000, max_tokens=0, n_tokens=0, n_streams=70000), -5)]
RINGS = [(dict(head_dim=48), -5), (dict(head_dim=288), -5), (dict(head_dim=0), -5), (dict(ring=ring(k_codes=None)), -1), (dict(ring=ring(v_scales=None)), -1), (dict(ring=ring(v_codes=AT + 8)), -5),
         (dict(slots=(1 << 24) + 1), -5)]


@pytest.mark.parametrize("kw,want", PACKING + RINGS + [
    (dict(heads_kv=0), -1), (dict(heads_kv=2000), -1), (dict(rotary_dim=66), -1), (dict(rotary_dim=7), -1), (dict(rotary_dim=-2), -1), (dict(slots=2), -1), (dict(sinks=-1), -1), (dict(eps=-1.0), -1),
    (dict(eps=NAN), -1), (dict(amplitude=INF), -1), (dict(k=toks(base=None)), -1), (dict(v=toks(base=AT + 2)), -1), (dict(frequencies=None), -1)])
def test_append_refuses(kw, want):
    refused("idf_nibble_append", append_args(**kw), want)


@pytest.mark.parametrize("kw,want", PACKING + RINGS + [
    (dict(heads_q=3), -1), (dict(heads_kv=0), -1), (dict(window=0), -1), (dict(sinks=-1), -1), (dict(slots=12), -1), (dict(window=12), -1), (dict(scale=0.0), -1), (dict(scale=NAN), -1), (dict(scale=INF), -1),
    (dict(q=toks(base=None)), -1), (dict(q=toks(base=AT + 8)), -5), (dict(out=toks(255)), -5), (dict(out=toks(128)), -1), (dict(out=toks(0, 0)), -1)])
def test_attend_refuses(kw, want):
    refused("idf_nibble_attend", attend_args(**kw), want)


def test_attend_wants_room_for_a_segment_beside_a_window():
    """Later tokens of a segment take the slots that earlier ones' windows lie in: not computed from what is there by then."""
    a, nb = attend_args(slots=2 + 8 + 3), C.c_size_t()
    assert idf.load_library().idf_nibble_attend_workspace(C.byref(a), C.byref(nb)) == 0
    refused("idf_nibble_attend", attend_args(slots=2 + 8 + 2), -1)


@pytest.mark.parametrize("kw,want", RINGS + [(dict(precision=2), -5), (dict(heads_kv=0), -1), (dict(n_streams=-1), -1), (dict(k=None), -1), (dict(v=AT + 4), -5), (dict(slots=0), -1)])
def test_values_refuse(kw, want):
    refused("idf_nibble_values", values_args(**kw), want)


GATES = PACKING + [(dict(channels=0), -5), (dict(channels=(1 << 20) + 1), -5), (dict(x=rows(base=None)), -1), (dict(gates=rows(base=None)), -1), (dict(gates=rows(base=AT + 2)), -1), (dict(x=rows(-64)), -5),
                   (dict(x=rows((1 << 25) + 1)), -5), (dict(marks=AT + 64), -1)]


@pytest.mark.parametrize("kw,want", GATES + [(dict(out=rows(63)), -1), (dict(out=rows(base=None)), -1), (dict(state_in=AT + 2), -1), (dict(n_tokens=4000, max_tokens=4000), -2)])
def test_gate_scan_refuses(kw, want):
    refused("idf_gate_scan", gate_args(**kw), want)


@pytest.mark.parametrize("kw,want", GATES + [(dict(grad_x=rows(63)), -1), (dict(grad_gates=rows(base=None)), -1), (dict(grad_out=rows(base=AT + 2)), -1), (dict(marks=None), -1), (dict(grad_state=AT + 2), -1),
                                             (dict(n_tokens=4000, max_tokens=4000), -2)])
def test_gate_scan_backward_refuses(kw, want):
    refused("idf_gate_scan_backward", back_args(**kw), want)


@pytest.mark.parametrize("fn", ["idf_quantize_rows", "idf_project_rows", "idf_nibble_append", "idf_nibble_attend", "idf_nibble_values", "idf_gate_scan", "idf_gate_scan_backward"])
def test_null_arguments(fn):
    refused(fn, None, -1)


def test_calls_without_rows_do_nothing():
    L = idf.load_library()
    for fn, a in (("idf_quantize_rows", quantize_args(n_rows=0, codes=None)), ("idf_project_rows", project_args(n_rows=0, weights=None)),
                  ("idf_nibble_append", append_args(n_tokens=0, max_tokens=0)), ("idf_nibble_attend", attend_args(n_tokens=0, max_tokens=0)),
                  ("idf_nibble_values", values_args(n_streams=0)), ("idf_gate_scan", gate_args(n_tokens=0, max_tokens=0)), ("idf_gate_scan_backward", back_args(n_tokens=0, max_tokens=0))):
        assert getattr(L, fn)(C.byref(a), None) == 0, fn


@pytest.mark.parametrize("call", [lambda x: idf.quantize_rows(x), lambda x: idf.project_rows(x, x.to(torch.int8), x[0]), lambda x: idf.gate_scan(x, x),
                                  lambda x: idf.nibble_attend(x[None], tokens.NibbleRing(*[x.to(torch.uint8)[None, None]] * 4), window=4),
                                  lambda x: idf.nibble_append(x[None], x[None], tokens.NibbleRing(*[x.to(torch.uint8)[None, None]] * 4)),
                                  lambda x: idf.nibble_values(tokens.NibbleRing(*[x.to(torch.uint8)[None, None]] * 4))])
def test_tensors_that_are_on_no_gpu(call):
    with pytest.raises(ValueError):
        call(torch.zeros(4, 64))


# ---- the oracle ----

def test_levels_and_ties():
    """Every border between two levels goes to the even code, what lies beside it to the nearer one; the power is the smallest that holds a block."""
    y = np.zeros((1, 32))
    y[0, :8] = [7, 5, 5 + 1e-9, 3.5, 2.5, 0.25, -0.75, -7]
    codes, powers = oracle.blocks(y)
    assert powers[0, 0] == 127 and codes[0, :8].tolist() == [7, 6, 7, 6, 4, 0, 10, 15]
    assert oracle.block_values(codes, powers)[0, :8].tolist() == [6, 4, 6, 4, 2, 0, -1, -6]
    y[0, 0] = np.nextafter(7, 8)
    assert oracle.blocks(y)[1][0, 0] == 128
    y[0, 3] = np.nan
    codes, powers = oracle.blocks(y)
    assert powers[0, 0] == 255 and not codes.any() and np.isnan(oracle.block_values(codes, powers)).all()
    assert oracle.blocks(np.zeros((1, 32)))[1][0, 0] == 27


def test_blocks_hold_what_they_hold():
    """Values of blocks come back as they are; nothing is off by more than half the widest step of a sixth of the largest value's power."""
    rng = np.random.default_rng(0)
    y = rng.standard_normal((50, 96)) * 2.0 ** rng.integers(-30, 30, (50, 1))
    codes, powers = oracle.blocks(y)
    v = oracle.block_values(codes, powers)
    again = oracle.blocks(v)
    assert np.array_equal(oracle.block_values(*again), v)
    assert np.all(np.abs(v - y) <= np.repeat(2.0 ** (powers.astype(float) - 127), 32, axis=-1))
    assert np.array_equal(torch.from_numpy(v).to(torch.bfloat16).double().numpy(), v)


def test_quantized_rows():
    codes, scales = oracle.quantize_rows(np.array([[127.0, 0.5, 1.5, -2.5, 0.0], [0, 0, 0, 0, 0], [1, np.inf, 0, 0, 0]]))
    assert codes.tolist() == [[127, 0, 2, -2, 0], [0] * 5, [0] * 5] and scales[0] == 1 and scales[1] == 0 and np.isnan(scales[2])


def test_gradients_against_differences():
    rng = np.random.default_rng(1)
    x, g, s, d, e = (rng.standard_normal(shape) for shape in ((6, 3), (6, 3), (3,), (6, 3), (3,)))

    def loss(x, g, s):
        h = oracle.gate_scan(x, g, s)[0]
        return (h * d).sum() + (h[-1] * e).sum()
    grads = oracle.gate_scan_backward(x, g, s, d, e)[:3]
    for i, grad in enumerate(grads):
        for at in np.ndindex(grad.shape):
            lo, hi = [[v.copy() for v in (x, g, s)] for _ in range(2)]
            hi[i][at] += 1e-5
            lo[i][at] -= 1e-5
            assert abs((loss(*hi) - loss(*lo)) / 2e-5 - grad[at]) <= 1e-8 * max(1, abs(grad[at]))


def test_recurrence_is_the_formula():
    rng = np.random.default_rng(2)
    x, g = rng.standard_normal((4, 2)), rng.standard_normal((4, 2))
    a = 1 / (1 + np.exp(-g))
    h = np.array([1.0, -2.0])
    hs = oracle.gate_scan(x, g, h)[0]
    for t in range(4):
        h = a[t] * h + (1 - a[t]) * x[t]
        assert np.allclose(hs[t], h, rtol=1e-14)


def test_matrices_that_share_places():
    """Against the set of all their places: columns beside each other, rows in between, one beginning within the other."""
    import random
    rng, seen = random.Random(3), set()
    buf = torch.zeros(400)
    for _ in range(3000):
        rows, cols, stride = rng.choice([1, 2, 5]), rng.choice([1, 3, 8]), rng.choice([8, 9, 17, 40])
        a, b = (buf.as_strided((rows, cols), (stride, 1), rng.randrange(0, 200)) for _ in range(2))
        places = [{t.storage_offset() + r * stride + c for r in range(rows) for c in range(cols)} for t in (a, b)]
        assert tokens._share(a, b) == bool(places[0] & places[1]), (rows, cols, stride, a.storage_offset(), b.storage_offset())
        seen.add(tokens._share(a, b))
    assert seen == {False, True}
    assert tokens._share(buf[:40].view(4, 10), buf[:60].view(4, 15)[:, :10]) and not tokens._share(buf[:40].view(4, 10), buf[40:100].view(4, 15)[:, :10])
    assert tokens._share(buf[:40].view(4, 10), buf[5:15].expand(4, 10)) and not tokens._share(buf[:0].view(0, 10), buf[:0].view(0, 10))
