"""The ring of 4-bit blocks: appending, what it stands for, and attention over it, against their definitions (oracle/few_bits.py, oracle/tokens.py).

Codes and powers are whole numbers and have to be equal; where keys are turned, float64 rounds an angle (position times frequency) and what is formed from it, so that a
code may differ where the value lies within 2^-40 of the middle between two.  Attention: the values that blocks stand for are exact, and the tolerance is that of attention
over a ring of such values (u half a step of the output's type, w = 2^-24): the output's rounding, in bfloat16 once more for the weights, scores and sums in float32.
"""
import numpy as np
import pytest
import torch

import paper_1804_10727_amd as idf
from oracle import few_bits, tokens as oracle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
W = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def normal(g, *shape, dtype):
    return torch.randn(shape, generator=g).to(dtype)


def within(got, want, bound, what=""):
    got = f64(got)
    assert got.shape == want.shape, what
    over = np.abs(got - want) / np.maximum(bound, 1e-300)
    assert np.all(np.isfinite(got)) and float(over.max(initial=0)) <= 1, f"{what}: {over.max(initial=0):.3g} of the bound at {np.unravel_index(over.argmax(), over.shape)}"


def alike(got, want, dtype, v):
    """Two ways to the same weights: in bfloat16 each of them is rounded or not, half a step 2^-9 of it, so that results are at most 2^-9 of the largest value apart before
    both are rounded; in float32 sums of 64 and of some hundred terms, of scores up to 20."""
    top = v.float().abs().max().item()
    return torch.allclose(got.float(), want.float(), rtol=torch.finfo(dtype).eps, atol=top * (2.0 ** -9 if dtype == torch.bfloat16 else 4 * 20 * 200 * W)) and bool(torch.isfinite(got).all())


def full_ring(streams, slots, heads, dim, byte=255):
    """A ring whose blocks are no numbers: nothing of them may show."""
    r = idf.nibble_ring(streams, slots, heads, dim, DEV)
    r.k_scales.fill_(byte)
    r.v_scales.fill_(byte)
    r.k_codes.fill_(0x5a)
    r.v_codes.fill_(0xa5)
    return r


def slot_of(p, sinks, slots):
    return p if p < sinks else sinks + (p - sinks) % (slots - sinks)


class Ring:
    """What a stream's ring has to hold, slot by slot: codes and powers of keys and values."""

    def __init__(self, slots, sinks, heads, dim):
        self.slots, self.sinks, self.held = slots, sinks, {}

    def append(self, start, k, v, exact=True):
        n, period = len(k), self.slots - self.sinks
        for t in range(n):
            p = start + t
            if p < self.sinks or t >= n - period:
                self.held[slot_of(p, self.sinks, self.slots)] = (few_bits.blocks(k[t]), few_bits.blocks(v[t]), k[t])

    def check(self, ring, b, turned=False, untouched=None):
        for s in range(self.slots):
            at = (b, slice(None), s)
            if s not in self.held:
                for got, was in zip(ring, untouched):
                    assert torch.equal(got[at], was[at]), f"slot {s} was not to be written"
                continue
            (kc, kp), (vc, vp), k = self.held[s]
            assert np.array_equal(few_bits.unpacked(ring.v_codes[at].cpu().numpy()), vc) and np.array_equal(ring.v_scales[at].cpu().numpy(), vp), f"values of slot {s}"
            assert np.array_equal(ring.k_scales[at].cpu().numpy(), kp), f"powers of keys of slot {s}"
            got = few_bits.unpacked(ring.k_codes[at].cpu().numpy())
            if not turned:
                assert np.array_equal(got, kc), f"keys of slot {s}"
                continue
            size = np.abs(k) / np.repeat(2.0 ** (kp.astype(float) - 127), 32, -1)
            borders = (few_bits.LEVELS[1:] + few_bits.LEVELS[:-1]) / 2
            near = np.abs(size[..., None] - borders).min(-1) < 2.0 ** -40
            assert np.all((got == kc) | near | ((size < 2.0 ** -40) & (got & 7 == kc & 7))), f"keys of slot {s}"


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("heads,dim,slots,sinks", [(1, 32, 9, 0), (3, 64, 16, 2), (2, 96, 40, 31), (8, 128, 12, 1), (2, 256, 5, 4), (5, 160, 30, 0)])
def test_append(heads, dim, slots, sinks, dtype):
    """Uneven segments, empty ones, ones longer than the ring, streams in another order; slots that nothing comes to stay."""
    g = torch.Generator().manual_seed(dim + slots)
    streams = 4
    ring = full_ring(streams, slots, heads, dim)
    was = [t.clone() for t in ring]
    refs, at = [Ring(slots, sinks, heads, dim) for _ in range(streams)], [0, 3, 1 << 33, sinks]
    for lengths, ids in (((1, 1, 1), (0, 2, 3)), ((0, 7, 50), (3, 0, 1)), ((3, 100, 2), (2, 1, 0)), ((4, 4, 4), (1, 2, 3))):
        n = sum(lengths)
        k, v = (normal(g, n, heads, dim, dtype=dtype) * torch.exp2(torch.randint(-20, 20, (n, heads, 1), generator=g).float()).to(dtype) for _ in range(2))
        offsets = torch.tensor([0] + list(lengths)).cumsum(0)
        idf.nibble_append(k.to(DEV), v.to(DEV), ring, torch.tensor([at[i] for i in ids], device=DEV), sinks=sinks, offsets=offsets.to(DEV), max_tokens=max(lengths),
                          stream_ids=torch.tensor(ids, dtype=torch.int32, device=DEV))
        for i, (a, m) in zip(ids, zip(offsets.tolist(), lengths)):
            refs[i].append(at[i], f64(k[a:a + m]), f64(v[a:a + m]))
            at[i] += m
    for b, r in enumerate(refs):
        r.check(ring, b, untouched=was)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim,rotary,weight", [(64, 64, True), (128, 64, False), (96, 20, True), (256, 256, True), (32, 6, False), (128, 0, True), (160, 34, True)])
def test_append_turns_and_normalises_keys(dim, rotary, weight, layout, dtype):
    g = torch.Generator().manual_seed(dim + rotary)
    n, heads, start = 23, 3, 100000
    packed = normal(g, n, 2 * heads * dim, dtype=dtype)
    k, v = packed[:, :heads * dim].unflatten(1, (heads, dim)), packed[:, heads * dim:].unflatten(1, (heads, dim))
    f = 10000.0 ** (-torch.arange(rotary // 2, dtype=torch.float64) / max(1, rotary // 2))
    w = 1 + 0.3 * torch.randn(dim, generator=g) if weight else None
    ring = full_ring(1, 30, heads, dim)
    was = [t.clone() for t in ring]
    on = packed.to(DEV)
    idf.nibble_append(on[:, :heads * dim].unflatten(1, (heads, dim)), on[:, heads * dim:].unflatten(1, (heads, dim)), ring, torch.tensor([start], device=DEV), frequencies=f.to(DEV) if rotary else None,
                      layout=layout, amplitude=1.25, k_weight=None if w is None else w.to(DEV), eps=1e-5)
    y = f64(k)
    if w is not None:
        y = f64(w) * y / np.sqrt(np.mean(y * y, axis=-1, keepdims=True) + 1e-5)
    for i in range(rotary // 2):
        a, b = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + rotary // 2)
        angle = ((start + np.arange(n)) * float(f[i]))[:, None]
        c, s = 1.25 * np.cos(angle), 1.25 * np.sin(angle)
        y[..., a], y[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    ref = Ring(30, 0, heads, dim)
    ref.append(start, y, f64(v))
    ref.check(ring, 0, turned=True, untouched=was)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_every_border(dtype):
    """Middles between levels and their neighbours in the type, with every power that a block can have; blocks of zeros, of the smallest and largest values, and
    with values that are not finite."""
    base = torch.zeros(64, dtype=torch.float32)
    middles = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    step = torch.finfo(dtype).eps
    base[:7], base[7:14], base[14:21] = middles, -middles * (1 + step), middles * (1 - step / 2)
    base[21], base[22:29] = 7.0, -middles
    base[32:39], base[39] = middles, 7.0 * (1 + step)
    tokens = [base * 2.0 ** e for e in range(-110, 126, 5)]
    special = torch.zeros(64)
    special[3], special[40] = float("nan"), 1.0
    tokens += [torch.zeros(64), special, special.clone().index_fill_(0, torch.tensor([3]), float("-inf")), base * 2.0 ** 125.2, base * 2.0 ** -126]
    x = torch.stack(tokens).to(dtype)[:, None]
    ring = full_ring(1, len(x), 1, 64)
    idf.nibble_append(x.to(DEV), x.flip(2).to(DEV), ring)
    ref = Ring(len(x), 0, 1, 64)
    with np.errstate(invalid="ignore", over="ignore"):
        ref.append(0, f64(x), f64(x.flip(2)))
        ref.check(ring, 0)
        k, v = idf.nibble_values(ring)
        for got, at in ((k, 0), (v, 1)):
            want = np.stack([few_bits.block_values(*ref.held[s][at]) for s in range(len(x))])
            assert np.array_equal(f64(got[0]), want, equal_nan=True)


@pytest.mark.parametrize("dim", [32, 96, 128, 256])
def test_values(dim):
    g = torch.Generator().manual_seed(dim)
    ring = idf.NibbleRing(*(torch.randint(lo, hi, (3, 2, 11, dim // by), generator=g, dtype=torch.uint8).to(DEV) for by, lo, hi in ((2, 0, 256), (32, 27, 253), (2, 0, 256), (32, 120, 130))))
    for dtype in (None, torch.float32, torch.bfloat16):
        k, v = idf.nibble_values(ring, dtype)
        assert k.dtype == (dtype or torch.bfloat16) and k.shape == (3, 11, 2, dim)
        for got, codes, scales in ((k, ring.k_codes, ring.k_scales), (v, ring.v_codes, ring.v_scales)):
            want = few_bits.block_values(few_bits.unpacked(codes.cpu().numpy()), scales.cpu().numpy())
            assert np.array_equal(f64(got), want.swapaxes(1, 2))


# ---- attention ----

def streams_through(dtype, hq, hkv, dim, window, sinks, room, pushes, seed=0, start=0, scale=None):
    g = torch.Generator().manual_seed(seed)
    streams, slots = len(pushes[0]), sinks + window + room
    scale = 1 / np.sqrt(dim) if scale is None else scale
    ring = full_ring(streams, slots, hkv, dim)
    ref = [oracle.Attention(window, sinks, scale, max(0, start - window)) for _ in range(streams)]

    def held(x):
        return few_bits.block_values(*few_bits.blocks(f64(x)))
    if start:
        old = [normal(g, streams * window, hkv, dim, dtype=dtype) for _ in range(2)]
        idf.nibble_append(*(x.to(DEV) for x in old), ring, torch.full((streams,), start - window, device=DEV), sinks=sinks)
        for b in range(streams):
            ref[b].push(np.zeros((window, hq, dim)), *(held(x[b * window:(b + 1) * window]) for x in old))
    u = 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2
    for lengths in pushes:
        n = sum(lengths)
        q, k, v = normal(g, n, hq, dim, dtype=dtype), normal(g, n, hkv, dim, dtype=dtype), normal(g, n, hkv, dim, dtype=dtype)
        starts = torch.tensor([r.p for r in ref], device=DEV)
        offsets = torch.tensor([0] + list(lengths)).cumsum(0)
        kw = dict(offsets=offsets.to(DEV), max_tokens=max(lengths), sinks=sinks)
        idf.nibble_append(k.to(DEV), v.to(DEV), ring, starts, **kw)
        out = idf.nibble_attend(q.to(DEV), ring, starts, window=window, scale=scale, **kw)
        for b in range(streams):
            s = slice(int(offsets[b]), int(offsets[b + 1]))
            want, size, score = ref[b].push(f64(q[s]), held(k[s]), held(v[s]))
            keys = min(ref[b].p, window + sinks)
            # (a weight below 2^-126 is none in float32, while blocks hold zeros: a result may be nothing but such weights' values)
            bound = torch.finfo(dtype).eps / 2 * np.abs(want) + (u + 2 * (2 * (dim + 8) * W * score[..., None] + (keys + 16) * W)) * size + keys * 2.0 ** -126 * np.abs(ref[b].v).max(initial=0)
            within(out[s], want, bound, f"stream {b} of {lengths} from {ref[b].p - lengths[b]}")
    return ring, ref


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("hq,hkv,dim,window,sinks", [(1, 1, 64, 1, 0), (4, 2, 64, 7, 2), (8, 1, 128, 64, 0), (3, 3, 96, 33, 5), (6, 2, 32, 100, 1), (2, 2, 160, 130, 64), (2, 1, 256, 40, 3), (32, 2, 128, 20, 4)])
def test_single_tokens(dtype, hq, hkv, dim, window, sinks):
    """From the first token on, past the point where the ring wraps."""
    pushes = [[1, 1, 1]] * 5 + [[60, 90, 1]] + [[1, 1, 1]] * 3 + [[64, 90, 31]] + [[1, 1, 1]] * 2
    streams_through(dtype, hq, hkv, dim, window, sinks, 89, pushes, seed=window)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("room", [299, 400])
@pytest.mark.parametrize("hq,hkv,dim,window,sinks", [(1, 1, 64, 1, 1), (4, 1, 32, 16, 0), (4, 4, 128, 65, 3), (10, 2, 96, 200, 70), (3, 1, 192, 31, 100), (2, 1, 256, 50, 2)])
def test_segments(dtype, hq, hkv, dim, window, sinks, room):
    """Uneven segments, empty ones, few tokens at a time, with just the room that they need."""
    pushes = [[0, 5, 17, 1], [130, 2, 0, 300], [9, 9, 9, 9], [1, 257, 40, 3], [0, 0, 1, 0]]
    streams_through(dtype, hq, hkv, dim, window, sinks, room, pushes, seed=window + dim)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("hq,hkv,dim", [(4, 1, 128), (2, 2, 64), (2, 1, 256)])
def test_long_windows_are_cut_into_parts(dtype, hq, hkv, dim):
    streams_through(dtype, hq, hkv, dim, 3000, 0, 60, [[1], [40], [1], [61]], seed=dim, start=1 << 33)
    streams_through(dtype, hq, hkv, dim, 1400, 5, 599, [[600]] * 3 + [[1], [40]], seed=dim)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_one_call_is_many_calls(dtype):
    """Since a token's keys are in the ring before it is asked for, how a stream is cut changes nothing but the order of sums."""
    g = torch.Generator().manual_seed(3)
    n, hq, hkv, dim = 200, 4, 2, 64
    q, k, v = (normal(g, n, h, dim, dtype=dtype).to(DEV) for h in (hq, hkv, hkv))
    outs = []
    for step in (200, 50, 7, 1):
        ring, got = full_ring(1, 20 + 3 + 200, hkv, dim), []
        for a in range(0, n, step):
            at = torch.tensor([a], device=DEV)
            idf.nibble_append(k[a:a + step], v[a:a + step], ring, at, sinks=3)
            got.append(idf.nibble_attend(q[a:a + step], ring, at, window=20, sinks=3))
        outs.append(torch.cat(got).float())
    for o in outs[1:]:
        assert torch.allclose(o, outs[0], rtol=0, atol=1e-5 if dtype == torch.float32 else 3 * 2 ** -8 * outs[0].abs().max().item())


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("tokens", [1, 3, 60])
def test_blocks_that_are_no_numbers(dtype, tokens):
    """Seen by a query they show in its row; where they are hidden nothing does, whatever other rows of the tile see."""
    g = torch.Generator().manual_seed(tokens)
    hkv, dim, window, n = 2, 64, 10, 40 + tokens
    q, k, v = normal(g, n, 4, dim, dtype=dtype), normal(g, n, hkv, dim, dtype=dtype), normal(g, n, hkv, dim, dtype=dtype)
    clean = full_ring(1, 150, hkv, dim)
    idf.nibble_append(k.to(DEV), v.to(DEV), clean)
    bad = idf.NibbleRing(*(t.clone() for t in clean))
    p = 40 + tokens // 2                                     # a key of head 0, a value of head 1
    bad.k_scales[0, 0, p, 1] = 255
    bad.v_scales[0, 1, p, 0] = 255
    start = torch.tensor([40], device=DEV)
    got, want = (idf.nibble_attend(q[40:].to(DEV), r, start, window=window) for r in (bad, clean))
    for t in range(tokens):
        sees = p <= 40 + t < p + window
        if not sees:
            assert alike(got[t], want[t], dtype, v)
            continue
        assert torch.isnan(got[t, :2]).all() and torch.isnan(got[t, 2:, :32]).all()
        assert alike(got[t, 2:, 32:], want[t, 2:, 32:], dtype, v)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_infinite_queries_stay_in_their_rows(dtype):
    g = torch.Generator().manual_seed(5)
    q, k, v = normal(g, 50, 4, 64, dtype=dtype), normal(g, 50, 2, 64, dtype=dtype), normal(g, 50, 2, 64, dtype=dtype)
    ring = full_ring(1, 100, 2, 64)
    idf.nibble_append(k.to(DEV), v.to(DEV), ring)
    want = idf.nibble_attend(q.to(DEV), ring, window=50)
    q[20, 1, 5], q[30, 2, 7] = float("inf"), float("nan")
    got = idf.nibble_attend(q.to(DEV), ring, window=50)
    rest = torch.ones(50, 4, dtype=torch.bool)
    rest[20, 1] = rest[30, 2] = False
    assert alike(got[rest], want[rest], dtype, v) and torch.isnan(got[30, 2]).all()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_large_scores(dtype):
    """Scores of thousands, and ones that are all alike."""
    streams_through(dtype, 2, 1, 64, 50, 1, 60, [[40], [1], [60]], seed=6, scale=40.0)
    ring = idf.nibble_ring(1, 64, 1, 64, DEV)
    g = torch.Generator().manual_seed(6)
    v = normal(g, 64, 1, 64, dtype=dtype)
    idf.nibble_append(torch.zeros_like(v).to(DEV), v.to(DEV), ring)
    out = idf.nibble_attend(torch.ones(1, 2, 64, dtype=dtype, device=DEV), ring, torch.tensor([63], device=DEV), window=64)
    mean = few_bits.block_values(*few_bits.blocks(f64(v[:, 0]))).mean(0)
    within(out[0, 0], mean, np.full(64, 80 * W) + torch.finfo(dtype).eps * (np.abs(mean) + 2.0 / 8), "mean")


def test_rows_that_no_segment_has_and_strange_places():
    """Negative starts, streams that are none, offsets that nobody meant: rows and rings of no segment stay as they are."""
    g = torch.Generator().manual_seed(7)
    q, k, v = (normal(g, 30, h, 64, dtype=torch.float32).to(DEV) for h in (2, 1, 1))
    ring = idf.nibble_ring(3, 60, 1, 64, DEV)
    was = [t.clone() for t in ring]
    for kw in (dict(starts=torch.tensor([-1, -(1 << 60), (1 << 62) + 1], device=DEV)), dict(starts=torch.zeros(3, dtype=torch.int64, device=DEV), stream_ids=torch.tensor([-1, 3, 1 << 30], dtype=torch.int32, device=DEV))):
        out = torch.full_like(q, 5.0)
        idf.nibble_append(k, v, ring, **kw)
        idf.nibble_attend(q, ring, window=20, out=out, **kw)
        assert torch.all(out == 5.0) and all(torch.equal(a, b) for a, b in zip(ring, was))
    for offsets in ([0, -7, 1 << 50, 30], [30, 20, 10, 0], [25, 99, 99, 99]):
        kw = dict(offsets=torch.tensor(offsets, device=DEV), max_tokens=30, starts=torch.tensor([0, 1 << 62, 5], device=DEV))
        idf.nibble_append(k, v, ring, **kw)
        idf.nibble_attend(q, ring, window=20, **kw)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_strides(dtype):
    g = torch.Generator().manual_seed(8)
    packed = normal(g, 33, 8 * 64 + 16, dtype=dtype).to(DEV)
    ring, other = idf.nibble_ring(1, 80, 2, 64, DEV), idf.nibble_ring(1, 80, 2, 64, DEV)
    for at in (0, 8, 3):
        q, k, v = packed[:, at:at + 256].unflatten(1, (4, 64)), packed[:, at + 256:at + 384].unflatten(1, (2, 64)), packed[:, at + 384:at + 512].unflatten(1, (2, 64))
        idf.nibble_append(k, v, ring)
        idf.nibble_append(k.contiguous(), v.transpose(0, 1).contiguous().transpose(0, 1), other)
        assert all(torch.equal(a, b) for a, b in zip(ring, other))
        out = torch.full((33, 6, 64), 4.0, dtype=dtype, device=DEV)
        got = idf.nibble_attend(q, ring, window=30, out=out[:, 1:5])
        assert torch.equal(got, idf.nibble_attend(q.contiguous(), ring, window=30)) and torch.all(out[:, 0] == 4.0) and torch.all(out[:, 5] == 4.0)


def test_recorded_steps_go_on_by_themselves():
    """Append and attend in one graph, positions read on the device, long enough windows to be cut; every replay against eager calls."""
    g = torch.Generator().manual_seed(9)
    rings = [idf.nibble_ring(2, 4 + 1500, 2, 128, DEV) for _ in range(2)]
    starts = [torch.full((2,), 1495, device=DEV) for _ in range(2)]
    f = idf.rotary_frequencies(128, device=DEV)[0]
    w = torch.ones(128, device=DEV)
    for r in rings:
        idf.nibble_append(*(normal(torch.Generator().manual_seed(1), 2 * 1495, 2, 128, dtype=torch.bfloat16).to(DEV) for _ in range(2)), r, torch.zeros(2, dtype=torch.int64, device=DEV), sinks=4)

    def step(i, q, k, v):
        idf.nibble_append(k, v, rings[i], starts[i], sinks=4, frequencies=f, k_weight=w)
        out = idf.nibble_attend(q, rings[i], starts[i], window=1500, sinks=4)
        starts[i] += 1
        return out
    still = [normal(g, 2, h, 128, dtype=torch.bfloat16).to(DEV) for h in (8, 2, 2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        spare = idf.nibble_ring(2, 4 + 1500, 2, 128, DEV)
        idf.nibble_append(still[1], still[2], spare, starts[0], sinks=4, frequencies=f, k_weight=w)
        idf.nibble_attend(still[0], spare, starts[0], window=1500, sinks=4)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(0, *still)
    for _ in range(20):
        new = [normal(g, 2, h, 128, dtype=torch.bfloat16).to(DEV) for h in (8, 2, 2)]
        want = step(1, *new)
        for s, x in zip(still, new):
            s.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(torch.equal(a, b) for a, b in zip(*rings))


def test_it_is_the_windows_attention_over_those_values():
    """The same as idf_window_attend over a ring of the values that the blocks stand for, up to the order of sums."""
    g = torch.Generator().manual_seed(10)
    q, k, v = (normal(g, 700, h, 128, dtype=torch.bfloat16).to(DEV) for h in (8, 2, 2))
    ring = idf.nibble_ring(1, 700, 2, 128, DEV)
    idf.nibble_append(k, v, ring)
    kk, vv = (x[0].contiguous() for x in idf.nibble_values(ring))
    a, b = idf.nibble_attend(q, ring, window=1).float(), idf.window_attend(q, kk, vv, window=1).float()
    assert torch.allclose(a, b, rtol=2 ** -7, atol=1e-6)
    assert idf.nibble_attend(q[:0], ring, torch.zeros(1, dtype=torch.int64, device=DEV), window=5).shape == (0, 8, 128)


def test_refusals_of_tensors():
    ring = idf.nibble_ring(2, 30, 2, 64, DEV)
    k, q, starts = torch.zeros(4, 2, 64, device=DEV), torch.zeros(4, 4, 64, device=DEV), torch.zeros(2, dtype=torch.int64, device=DEV)
    wrong = ring._replace(k_scales=ring.k_scales[:, :, :20].contiguous())
    for call in (lambda: idf.nibble_append(k, k[:, :1], ring, starts), lambda: idf.nibble_append(k, k.bfloat16(), ring, starts), lambda: idf.nibble_append(k[:3], k[:3], ring, starts), lambda: idf.nibble_append(k, k, wrong, starts),
                 lambda: idf.nibble_append(k, k, ring, starts.int()), lambda: idf.nibble_append(k, k, ring, starts, layout="pairs"), lambda: idf.nibble_append(k, k, ring, starts, k_weight=q[0, 0].double()),
                 lambda: idf.nibble_append(k, k, ring, starts, offsets=starts), lambda: idf.nibble_attend(q[..., :32], ring, starts, window=4), lambda: idf.nibble_attend(q, wrong, starts, window=4),
                 lambda: idf.nibble_attend(q.clone().requires_grad_(), ring, starts, window=4), lambda: idf.nibble_values(wrong), lambda: idf.nibble_values(ring, torch.float16), lambda: idf.nibble_ring(1, 4, 1, 48, DEV)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: idf.nibble_attend(q, ring, starts, window=30), lambda: idf.nibble_attend(q, ring, starts, window=4, sinks=30), lambda: idf.nibble_append(k, k, ring, starts, sinks=30),
                 lambda: idf.nibble_attend(torch.zeros(4, 3, 64, device=DEV), ring, starts, window=4), lambda: idf.nibble_attend(q, ring, starts, window=4, scale=0.0)):
        with pytest.raises(idf.IdfError):
            call()
