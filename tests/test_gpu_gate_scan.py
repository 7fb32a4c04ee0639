"""The gated recurrence and its gradients against their definitions in float64 (oracle/few_bits.py, pinned in test_few_bits_cpu.py).

Tolerances.  u is half a step of the output's type, w = 2^-24.  Outputs are rounded once: u |want|.  Every step's error is that of its gate (about ten
roundings and those of its exponent) and a few roundings of its terms, carried on as the state is: the oracle adds that up from the absolute terms.
"""
import numpy as np
import pytest
import torch

import paper_1804_10727_amd as idf
from oracle import few_bits as oracle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
W = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def within(got, want, bound, what=""):
    got = f64(got)
    assert got.shape == want.shape, what
    over = np.abs(got - want) / np.maximum(bound, 1e-300)
    assert np.all(np.isfinite(got)) and float(over.max(initial=0)) <= 1, f"{what}: {over.max(initial=0):.3g} of the bound at {np.unravel_index(over.argmax(), over.shape)}"


def make(lengths, channels, dtype, seed=0, open_=3.0):
    g = torch.Generator().manual_seed(seed)
    n = sum(lengths)
    x, gates = torch.randn(n, channels, generator=g).to(dtype), (torch.randn(n, channels, generator=g) * 2 + open_).to(dtype)
    state = torch.randn(len(lengths), channels, generator=g)
    d, end = torch.randn(n, channels, generator=g).to(dtype), torch.randn(len(lengths), channels, generator=g)
    return x, gates, state, d, end


def ragged(lengths):
    return dict(offsets=torch.tensor([0] + list(lengths)).cumsum(0).to(DEV), max_tokens=max(lengths))


def check(lengths, channels, dtype, seed=0, open_=3.0, even=False):
    x, gates, state, d, end = make(lengths, channels, dtype, seed, open_)
    kw = dict(n_segments=len(lengths)) if even else ragged(lengths)
    to = torch.full_like(state, float("nan")).to(DEV)
    gx, gg = x.to(DEV), gates.to(DEV)
    out, marks = idf.gate_scan(gx, gg, state.to(DEV), to, marks=True, **kw)
    grads = idf.gate_scan_backward(gx, gg, marks, d.to(DEV), end.to(DEV), **kw)
    u = torch.finfo(dtype).eps / 2
    at = 0
    for b, n in enumerate(lengths):
        s = slice(at, at + n)
        at += n
        hs, sizes, errors = oracle.gate_scan(f64(x[s]), f64(gates[s]), f64(state[b]))
        within(out[s], hs, u * np.abs(hs) + W * errors, f"out of segment {b}")
        within(to[b], hs[-1] if n else f64(state[b]), W * errors[-1] + 1e-30 if n else np.full(channels, 1e-30), f"state of segment {b}")
        dx, dg, ds, ex, eg, es = oracle.gate_scan_backward(f64(x[s]), f64(gates[s]), f64(state[b]), f64(d[s]), f64(end[b]))
        within(grads[0][s], dx, u * np.abs(dx) + W * ex + 1e-36, f"grad_x of segment {b}")
        within(grads[1][s], dg, u * np.abs(dg) + W * eg + 1e-36, f"grad_gates of segment {b}")
        within(grads[2][b], ds, W * es + 1e-30, f"grad_state of segment {b}")
    return out, to, grads


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("lengths", [(1,), (2, 0, 1), (15, 16, 17, 33), (300,), (1000, 0, 1, 517), (3000,)], ids=str)
@pytest.mark.parametrize("channels", [1, 2, 63, 128, 130, 321])
def test_segments(lengths, channels, dtype):
    """From single tokens to segments that are cut into parts, channels that fill no wave, states of their own."""
    check(lengths, channels, dtype, seed=channels)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("open_", [-6.0, 0.0, 9.0])
def test_gates_that_are_shut_or_open(dtype, open_):
    check((700, 64), 192, dtype, seed=5, open_=open_)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_segments_of_one_length(dtype):
    check((200,) * 3, 64, dtype, even=True)
    check((1,) * 70, 96, dtype, even=True)


@pytest.mark.parametrize("n", [16, 200, 20000])
def test_a_state_that_is_what_comes_in_stays(n):
    """Gates that keep nearly everything, and values equal to the state: what is kept, rounded by itself to a number near one, would move it.  A part from
    nothing is rounded at every step, half a step each."""
    x, gates = torch.full((n, 64), 0.37, device=DEV), torch.full((n, 64), 12.0, device=DEV)
    out = idf.gate_scan(x, gates, x[:1].contiguous())
    assert torch.equal(out, x) if n == 16 else (out - x).abs().max() <= 2 * 2048 * W * 0.37       # (16 tokens are never cut)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_cuts_agree_and_runs_repeat(dtype):
    """A segment in one call, in three calls with its state handed on, and among others: the same within the bound; twice the same: the same bits."""
    x, gates, state, d, end = (t.to(DEV) for t in make((2500,), 128, dtype, seed=9))
    to = torch.empty_like(state)
    out = idf.gate_scan(x, gates, state, to)
    again = idf.gate_scan(x, gates, state, torch.empty_like(state))
    assert torch.equal(out, again)
    s = state.clone()
    pieces = [idf.gate_scan(x[a:b], gates[a:b], s, s) for a, b in ((0, 700), (700, 701), (701, 2500))]
    hs, _, errors = oracle.gate_scan(f64(x), f64(gates), f64(state[0]))
    within(torch.cat(pieces), hs, torch.finfo(dtype).eps / 2 * np.abs(hs) + W * errors)
    within(s[0], hs[-1], W * errors[-1])
    assert torch.allclose(s, to, rtol=1e-5, atol=1e-6)


def test_state_in_place_while_segments_are_cut():
    """state_out is state: the last part of a segment writes what its first one begins with, grad_state in the same way."""
    x, gates, state, d, end = (t.to(DEV) for t in make((20000, 20000), 64, torch.float32, seed=2, open_=9.0))
    for _ in range(5):
        s, to = state.clone(), torch.empty_like(state)
        kw = dict(n_segments=2)
        assert torch.equal(idf.gate_scan(x, gates, s, s, **kw), idf.gate_scan(x, gates, state, to, **kw)) and torch.equal(s, to)


def test_streams_by_ids_and_segments_of_none():
    """Segments of any order of streams; one whose stream is none takes no part: its rows and the state stay, its gradients are zero."""
    lengths, streams = (40, 5, 33, 0), 6
    x, gates, _, d, _ = make(lengths, 70, torch.float32, seed=3)
    state = torch.randn(streams, 70, generator=torch.Generator().manual_seed(4))
    for ids in ([4, 0, 5, 1], [4, -1, 5, 1], [4, 99, 5, 1]):
        kw = dict(stream_ids=torch.tensor(ids, dtype=torch.int32, device=DEV), **ragged(lengths))
        s, out = state.clone().to(DEV), torch.full(x.shape, 7.0, device=DEV)
        _, marks = idf.gate_scan(x.to(DEV), gates.to(DEV), s, s, out=out, marks=True, **kw)
        end = torch.randn(streams, 70, generator=torch.Generator().manual_seed(5)).to(DEV)
        dx, dg, ds = idf.gate_scan_backward(x.to(DEV), gates.to(DEV), marks, d.to(DEV), end, **kw)
        at = 0
        for n, b in zip(lengths, ids):
            rows = slice(at, at + n)
            at += n
            if not 0 <= b < streams:
                assert torch.all(out[rows] == 7.0) and not dx[rows].any() and not dg[rows].any()
                continue
            hs, _, errors = oracle.gate_scan(f64(x[rows]), f64(gates[rows]), f64(state[b]))
            within(out[rows], hs, W * (errors + np.abs(hs)))
            within(s[b], hs[-1] if n else f64(state[b]), W * errors[-1] + 1e-30 if n else np.full(70, 1e-30))
            want = oracle.gate_scan_backward(f64(x[rows]), f64(gates[rows]), f64(state[b]), f64(d[rows]), f64(end[b]))
            within(ds[b], want[2], W * want[5] + 1e-30)
        untouched = [b for b in range(streams) if b not in ids]
        assert torch.equal(s[untouched].cpu(), state[untouched])


def test_rows_that_no_segment_has():
    """In front of the first segment, behind the last one, beyond max_tokens: results stay as they were, gradients are zero."""
    x, gates, _, d, _ = (t.to(DEV) for t in make((50,), 33, torch.float32, seed=6))
    kw = dict(offsets=torch.tensor([5, 20, 20, 40], device=DEV), max_tokens=12)
    out = torch.full_like(x, 3.0)
    _, marks = idf.gate_scan(x, gates, out=out, marks=True, **kw)
    dx, dg, _ = idf.gate_scan_backward(x, gates, marks, d, **kw)
    mine = torch.zeros(50, dtype=torch.bool)
    mine[5:17] = mine[20:32] = True
    assert torch.all(out[~mine] == 3.0) and not dx[~mine].any() and not dg[~mine].any()
    for a in (5, 20):
        hs, _, errors = oracle.gate_scan(f64(x[a:a + 12]), f64(gates[a:a + 12]), np.zeros(33))
        within(out[a:a + 12], hs, W * (errors + np.abs(hs)))


@pytest.mark.parametrize("offsets", [[0, -5, 30], [10, 5, 1 << 40], [0, 99, 20]])
def test_offsets_that_nobody_meant_stay_in_bounds(offsets):
    x, gates, _, d, _ = (t.to(DEV) for t in make((30,), 64, torch.float32))
    guard = torch.full((32, 64), 5.0, device=DEV)
    kw = dict(offsets=torch.tensor(offsets, device=DEV), max_tokens=30)
    _, marks = idf.gate_scan(x, gates, out=guard[1:31], marks=True, **kw)
    idf.gate_scan_backward(x, gates, marks, d, **kw)
    torch.cuda.synchronize()
    assert torch.all(guard[0] == 5.0) and torch.all(guard[31] == 5.0)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_strides_and_alignment(dtype):
    """Columns of a wider matrix from an odd place on, rows that repeat, an out among other columns."""
    g = torch.Generator().manual_seed(7)
    wide = torch.randn(90, 200, generator=g).to(dtype).to(DEV)
    for first, channels in ((0, 64), (3, 64), (1, 33), (2, 66)):
        x, gates = wide[:, first:first + channels], wide[:, 100 + first:100 + first + channels]
        to = torch.full((90, 150), 9.0, dtype=dtype, device=DEV)
        got, marks = idf.gate_scan(x, gates, out=to[:, first:first + channels], marks=True)
        want = idf.gate_scan(x.contiguous(), gates.contiguous())
        assert torch.equal(got, want) and torch.all(to[:, :first] == 9.0) and torch.all(to[:, first + channels:] == 9.0)
        a = idf.gate_scan_backward(x, gates, marks, wide[:, 50:50 + channels])
        b = idf.gate_scan_backward(x.contiguous(), gates.contiguous(), marks, wide[:, 50:50 + channels].contiguous())
        assert all(torch.equal(s, t) for s, t in zip(a, b))
    row = wide[:1, :64].expand(90, 64)
    assert torch.equal(idf.gate_scan(row, wide[:, 64:128]), idf.gate_scan(row.contiguous(), wide[:, 64:128].contiguous()))
    assert torch.equal(idf.gate_scan(wide.t()[:64, :50], wide.t()[64:128, :50]), idf.gate_scan(wide.t()[:64, :50].contiguous(), wide.t()[64:128, :50].contiguous()))


@pytest.mark.parametrize("n", [40, 3000])
def test_what_is_infinite_or_not_a_number(n):
    """An infinite value stays in the state, with its sign; what is not a number stays that; other channels see nothing of either."""
    x, gates, state, d, end = make((n,), 64, torch.float32, seed=8)
    inf, nan = float("inf"), float("nan")
    x[n // 2, 3], x[n // 3, 5], x[n // 2, 5], x[7, 9], gates[n // 2, 11] = inf, -inf, -inf, nan, nan
    x[n // 4, 13], x[n // 2, 13] = inf, -inf
    gates[:, 15], gates[:, 17] = inf, -inf
    state[0, 21] = -inf
    to = torch.empty(1, 64, device=DEV)
    out = idf.gate_scan(x.to(DEV), gates.to(DEV), state.to(DEV), to)
    with np.errstate(invalid="ignore", over="ignore"):
        hs, _, errors = oracle.gate_scan(f64(x), f64(gates), f64(state[0]))
    got = f64(out)
    fine = np.isfinite(hs)
    assert np.array_equal(np.isnan(hs), np.isnan(got)) and np.array_equal(hs[~fine & ~np.isnan(hs)], got[~fine & ~np.isnan(hs)])
    assert np.all(np.abs(got - hs)[fine] <= (W * (errors + np.abs(hs)))[fine]) and np.array_equal(got[-1], f64(to[0]), equal_nan=True)


def test_an_infinite_gradient_stays_in_its_channel():
    n = 2500
    x, gates, state, d, end = make((n,), 64, torch.float32, seed=10)
    _, marks = idf.gate_scan(x.to(DEV), gates.to(DEV), state.to(DEV), marks=True)
    want = idf.gate_scan_backward(x.to(DEV), gates.to(DEV), marks, d.to(DEV), end.to(DEV))
    bad = d.clone()
    bad[n // 2, 3], bad[n - 1, 9] = float("inf"), float("nan")
    got = idf.gate_scan_backward(x.to(DEV), gates.to(DEV), marks, bad.to(DEV), end.to(DEV))
    others = [c for c in range(64) if c not in (3, 9)]
    assert all(torch.equal(a[:, others], b[:, others]) for a, b in zip(got, want))
    assert torch.all(torch.isinf(got[0][:n // 2 + 1, 3])) and torch.equal(got[0][n // 2 + 1:, 3], want[0][n // 2 + 1:, 3]) and torch.isinf(got[2][0, 3])
    assert torch.all(torch.isnan(got[0][:, 9]))


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_recorded_by_torch(dtype):
    """gate_scan_recorded with torch's gradients, for the result, the end, or both of them, and for some of the leaves only."""
    lengths = (37, 0, 150)
    x, gates, state, d, end = (t.to(DEV) for t in make(lengths, 66, dtype, seed=11))
    kw = ragged(lengths)
    out, marks = idf.gate_scan(x, gates, state, marks=True, **kw)
    for use_out, use_end in ((True, True), (True, False), (False, True)):
        want = idf.gate_scan_backward(x, gates, marks, d if use_out else None, end if use_end else None, n_streams=3, **kw)
        leaves = [t.clone().requires_grad_() for t in (x, gates, state)]
        got, ends = idf.gate_scan_recorded(*leaves, **kw)
        assert torch.equal(got, out)
        torch.autograd.backward([t for t, use in ((got, use_out), (ends, use_end)) if use], [t for t, use in ((d, use_out), (end, use_end)) if use])
        assert all(torch.equal(a.grad, b) for a, b in zip(leaves, want))
    g = gates.clone().requires_grad_()
    got, ends = idf.gate_scan_recorded(x, g, None, **kw)
    (got.float().sum() + ends.sum()).backward()
    assert g.grad is not None and torch.isfinite(g.grad).all()
    (dg,) = torch.autograd.grad(idf.gate_scan_recorded(x, g)[0].float().sum(), g, create_graph=True)
    with pytest.raises(RuntimeError):
        dg.float().sum().backward()


def test_shared_and_broadcast_leaves():
    """A gate per channel that all tokens share, and x that is the gate as well: torch adds the gradients up."""
    x, gates, _, d, _ = (t.to(DEV) for t in make((120,), 64, torch.float32, seed=12))
    one = gates[0].clone().requires_grad_()
    idf.gate_scan_recorded(x, one.expand(120, 64))[0].backward(d)
    _, marks = idf.gate_scan(x, gates[:1].expand(120, 64), marks=True)
    want = idf.gate_scan_backward(x, gates[:1].expand(120, 64), marks, d)
    assert torch.allclose(one.grad, want[1].sum(0), rtol=1e-4, atol=1e-5)
    y = x.clone().requires_grad_()
    idf.gate_scan_recorded(y, y)[0].backward(d)
    _, marks = idf.gate_scan(x, x, marks=True)
    want = idf.gate_scan_backward(x, x, marks, d)
    assert torch.equal(y.grad, want[0] + want[1])


def test_recorded_into_a_graph():
    """Both passes in one graph, replayed on other inputs with eager work between; the call that torch records is refused there, in either pass."""
    x, gates, state, d, end = (t.to(DEV) for t in make((900, 900), 128, torch.bfloat16, seed=13))
    kw = dict(n_segments=2)
    leaf = x.clone().requires_grad_()
    alive, _ = idf.gate_scan_recorded(leaf, gates, state, **kw)            # an eager graph of the same leaves lives
    sx, sd, st = x.clone(), d.clone(), state.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _, m = idf.gate_scan(sx, gates, st.clone(), marks=True, **kw)
        idf.gate_scan_backward(sx, gates, m, sd, end, **kw)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, marks = idf.gate_scan(sx, gates, st, st, marks=True, **kw)
        grads = idf.gate_scan_backward(sx, gates, marks, sd, end, **kw)
        with pytest.raises(RuntimeError, match="captured"):
            idf.gate_scan_recorded(leaf, gates, state, **kw)
    want_state = state.clone()
    for i in range(4):
        sx.copy_(x * (1 + i))
        sd.copy_(d.flip(0) if i % 2 else d)
        before = want_state.clone()
        want, m = idf.gate_scan(sx, gates, before, want_state, marks=True, **kw)
        want_grads = idf.gate_scan_backward(sx, gates, m, sd, end, **kw)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(st, want_state) and all(torch.equal(a, b) for a, b in zip(grads, want_grads))
    alive.backward(d)
    assert torch.isfinite(leaf.grad).all()


def test_on_a_stream_of_its_own():
    x, gates, state, d, end = (t.to(DEV) for t in make((5000,), 256, torch.bfloat16, seed=14))
    want = idf.gate_scan(x, gates, state)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        outs = [idf.gate_scan(x, gates, state) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("long_first", [True, False])
def test_one_long_segment_among_many_short_ones(dtype, long_first):
    """Summaries lie by the tokens before a segment: none of them lies on another's, wherever the long segment stands and ends."""
    short = [i * 7 % 5 for i in range(90)] + [16, 32, 31, 160, 161, 0, 0]
    check([2500] + short if long_first else short + [2500, 1, 0, 1100, 3], 70, dtype, seed=21)


@pytest.mark.parametrize("offsets", [[0, -5, 4000, 1000, 6000], [6000, 5, 3000, 1 << 40, 0], [0, 5999, 20, 5990, 300], [4000, 4000, 10, 10, 6000], [-1] * 5, [1 << 62] * 5],
                         ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_offsets_that_nobody_meant_end_in_bounds(offsets, dtype):
    """Tiles of long segments wait for each other: whatever the offsets say, they all end, and nothing beside the rows is written."""
    x, gates, _, d, _ = (t.to(DEV) for t in make((6000,), 192, dtype))
    guard = torch.full((6002, 192), 5.0, dtype=dtype, device=DEV)
    kw = dict(offsets=torch.tensor(offsets, device=DEV), max_tokens=6000)
    _, marks = idf.gate_scan(x, gates, out=guard[1:6001], marks=True, **kw)
    idf.gate_scan_backward(x, gates, marks, d, **kw)
    torch.cuda.synchronize()
    assert torch.all(guard[0] == 5.0) and torch.all(guard[6001] == 5.0)


def test_long_segments_of_no_stream_and_rows_of_no_segment():
    """A stream that is none between others, bounds shorter than what the offsets leave, empty segments: tiles that have nothing to do hold up nobody."""
    lengths, streams = (2500, 0, 3000, 1, 2600), 5
    x, gates, _, d, _ = (t.to(DEV) for t in make((9000,), 70, torch.float32, seed=31))
    state, end = (torch.randn(streams, 70, generator=torch.Generator().manual_seed(s)).to(DEV) for s in (32, 33))
    offsets = torch.tensor([100, 2700, 2700, 5800, 5801, 8500], device=DEV)
    for ids in ([4, 0, 2, 1, 3], [4, 0, -1, 1, 3], [-7, 0, 2, 99, 3]):
        kw = dict(stream_ids=torch.tensor(ids, dtype=torch.int32, device=DEV), offsets=offsets, max_tokens=3000)
        s, out = state.clone(), torch.full_like(x, 7.0)
        _, marks = idf.gate_scan(x, gates, s, s, out=out, marks=True, **kw)
        dx, dg, ds = idf.gate_scan_backward(x, gates, marks, d, end, **kw)
        mine = torch.zeros(9000, dtype=torch.bool)
        for i, b in enumerate(ids):
            rows = slice(int(offsets[i]), min(int(offsets[i + 1]), int(offsets[i]) + 3000))
            if not 0 <= b < streams:
                continue
            mine[rows] = True
            hs, _, errors = oracle.gate_scan(f64(x[rows]), f64(gates[rows]), f64(state[b]))
            within(out[rows], hs, W * (errors + np.abs(hs)))
            want = oracle.gate_scan_backward(f64(x[rows]), f64(gates[rows]), f64(state[b]), f64(d[rows]), f64(end[b]))
            for got, w, e in ((dx[rows], want[0], want[3]), (dg[rows], want[1], want[4]), (ds[b], want[2], want[5])):
                within(got, w, W * (np.abs(w) + e) + 1e-30)
            within(s[b], hs[-1] if len(hs) else f64(state[b]), W * errors[-1] + 1e-30 if len(hs) else np.full(70, 1e-30))
        assert torch.all(out[~mine] == 7.0) and not dx[~mine].any() and not dg[~mine].any()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_numbers_of_all_ones(dtype):
    """Not numbers whose bits are all set, in values, gates, states and gradients: as any other that is not a number."""
    n = 3000
    x, gates, state, d, end = (t.to(DEV) for t in make((n,), 128, dtype, seed=34))
    want = idf.gate_scan(x, gates, state)
    ones = torch.full((1,), -1, dtype=torch.int32 if dtype == torch.float32 else torch.int16, device=DEV).view(dtype)
    x[5, 3], gates[700, 9], d[2000, 20] = ones[0], ones[0], ones[0]
    state[0, 15], end[0, 17] = (torch.full((1,), -1, dtype=torch.int32, device=DEV).view(torch.float32)[0] for _ in range(2))
    to = torch.empty_like(state)
    out, marks = idf.gate_scan(x, gates, state, to, marks=True)
    dx, dg, ds = idf.gate_scan_backward(x, gates, marks, d, end)
    bad = torch.zeros(n, 128, dtype=torch.bool, device=DEV)
    bad[5:, 3] = bad[700:, 9] = bad[:, 15] = True
    assert torch.equal(torch.isnan(out), bad) and torch.equal(out[~bad], want[~bad]) and torch.equal(torch.isnan(to[0]), bad[-1])
    nan = torch.isnan(ds[0])
    assert nan[9] and nan[20] and nan[17] and int(nan.sum()) == 3
    assert torch.isnan(dx[:2001, 20]).all() and not torch.isnan(dx[2001:, 20]).any() and torch.isnan(dx[:, 17]).all()


def test_two_calls_at_once():
    """Tiles of two calls on two streams are on the machine together, more of them than it holds: each waits for its own call's only."""
    sets = [tuple(t.to(DEV) for t in make((9000, 7000), 1024, torch.bfloat16, seed=s)) for s in (35, 36)]
    kw = ragged((9000, 7000))

    def both(x, gates, state, d, end):
        to = torch.empty_like(state)
        out, marks = idf.gate_scan(x, gates, state, to, marks=True, **kw)
        return (out, to, *idf.gate_scan_backward(x, gates, marks, d, end, **kw))
    want = [both(*s) for s in sets]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(both(*sets[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in range(2) for run in got[i] for a, b in zip(run, want[i]))


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("lengths", [(4096 + 1,), (8192 * 2 + 255, 1, 4095), (128, 129, 255, 256, 257, 2047, 2048, 2049)], ids=str)
def test_segments_that_end_about_a_tile(lengths, dtype):
    """Ends at, before and behind the borders of waves, tiles and of the rows that a state is told for."""
    check(lengths, 66, dtype, seed=37)


def test_out_that_shares_places_is_refused():
    """The result over x or gates is refused; beside them in one matrix it is taken."""
    both = torch.randn(300, 192, generator=torch.Generator().manual_seed(40)).to(DEV)
    x, gates, out = both[:, :64], both[:, 64:128], both[:, 128:]
    want = idf.gate_scan(x, gates)
    assert idf.gate_scan(x, gates, out=out) is out and torch.equal(out, want)
    for bad in (x, gates, both[:, 32:96], both[:, 1:65]):
        with pytest.raises(ValueError, match="shares"):
            idf.gate_scan(x, gates, out=bad)
    with pytest.raises(ValueError, match="shares"):
        y = both[:, :64].contiguous()
        idf.gate_scan(y, y, out=y)


def test_streams_that_no_segment_is_of_have_no_gradient():
    x, gates, _, d, _ = (t.to(DEV) for t in make((40,), 32, torch.float32, seed=41))
    _, marks = idf.gate_scan(x, gates, marks=True)
    for kw in (dict(n_streams=5), dict(n_streams=5, stream_ids=torch.tensor([3], dtype=torch.int32, device=DEV))):
        at = 3 if "stream_ids" in kw else 0
        filler = torch.full((5, 32), float("nan"), device=DEV)
        del filler                                 # (its memory is likely to be taken next)
        ds = idf.gate_scan_backward(x, gates, marks, d, n_segments=1, **kw)[2]
        assert ds.shape == (5, 32) and ds[at].any() and not ds[[i for i in range(5) if i != at]].any()


@pytest.mark.parametrize("lengths,front,behind", [((1, 1, 0, 1), 5, 3000), ((40, 0, 17), 900, 2000), ((700, 3, 0, 500), 300, 0), ((700, 3, 0, 500), 1000, 5000), ((128,), 0, 1), ((129,), 127, 129)])
def test_padded_batches(lengths, front, behind):
    """Many rows in front of the first segment and behind the last one, and behind segments that are cut at max_tokens: no gradient, whichever workgroup clears them."""
    n = front + sum(lengths) + behind
    x, gates, _, d, _ = (t.to(DEV) for t in make((n,), 130, torch.bfloat16, seed=50))
    offsets = (front + torch.tensor([0] + list(lengths)).cumsum(0)).to(DEV)
    for longest in (max(lengths), max(1, max(lengths) - 200)):
        kw = dict(offsets=offsets, max_tokens=longest)
        _, marks = idf.gate_scan(x, gates, marks=True, **kw)
        filler = [torch.full_like(x, float("nan")) for _ in range(2)]
        del filler                                 # (their memory is likely to be taken for the gradients)
        dx, dg, _ = idf.gate_scan_backward(x, gates, marks, d, **kw)
        mine = torch.zeros(n, dtype=torch.bool)
        for b, length in enumerate(lengths):
            mine[int(offsets[b]):int(offsets[b]) + min(length, longest)] = True
        assert not dx[~mine].any() and not dg[~mine].any() and dx[mine].any(1).all() and torch.isfinite(dg).all()
