"""The operators that mix the tokens of streams against their definitions in float64 (oracle/tokens.py).

Tolerances.  u is half a step of the output's type (eps / 2), w = 2^-24 that of float32.  Outputs are rounded once: u |want|.  Products of
sums on the matrix cores take rounded factors in bfloat16 (softmax weights; scores and states of the linear attention): another u times the sum of
absolute terms, twice where two factors on the way are rounded.  Float32 sums of n terms are off by at most n w times the sum of absolute terms,
a score's error is one of the weight's exponent, a power of a decay is off by its exponent times w; each of those counted twice, for
the other roundings on the way (scaling, exponential, reciprocal).
"""
import numpy as np
import pytest
import torch

import paper_1804_10727_amd as idf
from oracle import tokens as oracle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
W = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]


def half_step(t):
    return torch.finfo(t).eps / 2


def rounded(t):
    return 0.0 if t == torch.float32 else half_step(t)


def normal(g, *shape, dtype):
    return torch.randn(shape, generator=g).to(dtype)


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def within(got, want, bound, what=""):
    got = f64(got)
    assert got.shape == want.shape, what
    over = np.abs(got - want) / np.maximum(bound, 1e-300)
    fine = bool(np.all(np.isfinite(got))) and float(over.max(initial=0)) <= 1
    assert fine, f"{what}: {over.max(initial=0):.3g} of the bound at {np.unravel_index(over.argmax(), over.shape)}"


# ---- norms and rotation ----

@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("n,hq,hk,d,r", [(1, 1, 1, 64, 64), (7, 5, 1, 128, 128), (33, 4, 2, 96, 32), (5, 3, 3, 80, 20), (3, 2, 1, 256, 256), (9, 1, 2, 18, 6),
                                         (130, 16, 4, 64, 16), (4, 2, 2, 255, 250), (2, 40, 8, 128, 0), (3, 0, 2, 32, 32), (1100, 2, 1, 32, 32), (3, 3, 1, 1, 0)])
def test_norm_rotate(n, hq, hk, d, r, layout, dtype):
    g = torch.Generator().manual_seed(n * 1000 + d)
    q, k = normal(g, n, hq, d, dtype=dtype), normal(g, n, hk, d, dtype=dtype)
    positions = torch.randint(0, 1 << 24, (n,), generator=g)
    positions[0] = 0
    frequencies = 10000.0 ** (-torch.arange(r // 2, dtype=torch.float64) / max(1, r // 2))
    qw, kw = 1 + 0.3 * torch.randn(d, generator=g), None
    got = idf.norm_rotate(q.to(DEV), k.to(DEV), positions.to(DEV), frequencies.to(DEV), layout=layout, amplitude=1.25, q_weight=qw.to(DEV), eps=1e-5)
    for out, x, weight in zip(got, (q, k), (qw, kw)):
        assert out.dtype == dtype and out.shape == x.shape
        want, size = oracle.norm_rotate(f64(x), positions.numpy(), frequencies.numpy(), layout == "interleaved", 1.25, None if weight is None else f64(weight), 1e-5)
        # the sum of squares by d terms, root, quotient, weight, cosine, products: each a float32 rounding (the cosine's argument too)
        within(out, want, half_step(dtype) * np.abs(want) + 2 * (d + 16) * W * size, f"{x.shape}")


def test_norm_rotate_in_place_of_strided_views():
    """Views of one projection, written where they were read; what lies between them stays."""
    g = torch.Generator().manual_seed(3)
    packed = normal(g, 50, 6 * 64 + 24, dtype=torch.bfloat16).to(DEV)
    for first, why in ((0, "aligned"), (5, "not aligned"), (2, "by pairs")):
        x = packed.clone()
        q, k = x[:, first:first + 4 * 64].unflatten(1, (4, 64)), x[:, first + 4 * 64:first + 6 * 64].unflatten(1, (2, 64))
        positions = torch.arange(50, device=DEV) + 1000
        f, amplitude = idf.rotary_frequencies(64, device=DEV)
        w = torch.full((64,), 0.5, device=DEV)
        want = idf.norm_rotate(q.contiguous(), k.contiguous(), positions, f, amplitude=amplitude, q_weight=w, k_weight=w)
        a, b = idf.norm_rotate(q, k, positions, f, amplitude=amplitude, q_weight=w, k_weight=w, q_out=q, k_out=k)
        assert a is q and b is k
        # another way to cut a head into pieces adds its squares in another order: a last bit of the norm may differ
        for x_, y_ in zip((q, k), want):
            assert torch.allclose(x_.float(), y_.float(), rtol=2 ** -7, atol=1e-6), why
        assert torch.equal(x[:, :first], packed[:, :first]) and torch.equal(x[:, first + 6 * 64:], packed[:, first + 6 * 64:])


def test_norm_rotate_heads_first_and_many_tokens():
    """Tokens that lie behind each other per head, an empty set of them, and rows of zeros."""
    g = torch.Generator().manual_seed(4)
    q = normal(g, 3, 700, 64, dtype=torch.float32).to(DEV).transpose(0, 1)
    k = torch.zeros(700, 1, 64, device=DEV)
    f, _ = idf.rotary_frequencies(64, scaling="parts", factor=8.0, device=DEV)
    positions = torch.arange(700, device=DEV)
    w = torch.ones(64, device=DEV)
    a, b = idf.norm_rotate(q, k, positions, f, q_weight=w, k_weight=w)
    want = idf.norm_rotate(q.contiguous(), k, positions, f, q_weight=w, k_weight=w)
    assert torch.equal(a, want[0]) and torch.equal(b, torch.zeros_like(k))
    a, b = idf.norm_rotate(q[:0], k[:0], positions[:0], f)
    assert a.shape == (0, 3, 64) and b.shape == (0, 1, 64)


# ---- attention over a window ----

def window_streams(dtype, hq, hkv, d, window, sinks, room, pushes, seed=0, ragged=True, start=0, scale=None):
    """Streams pushed segment by segment: pushes is a list of lists of lengths, one length per stream.  Rings begin full of NaN, which
    no query may see."""
    g = torch.Generator().manual_seed(seed)
    streams = len(pushes[0])
    scale = 1 / np.sqrt(d) if scale is None else scale
    rings = [torch.full((streams, sinks + window + room, hkv, d), float("nan"), dtype=dtype, device=DEV) for _ in range(2)]
    ref = [oracle.Attention(window, sinks, scale, max(0, start - window)) for _ in range(streams)]
    for b in range(streams if start else 0):                            # what came before: the ring holds it, the oracle was given it
        old = [normal(g, window, hkv, d, dtype=dtype) for _ in range(2)]
        slots = sinks + (torch.arange(start - window, start) - sinks) % (window + room)
        for r, x in zip(rings, old):
            r[b, slots.to(DEV)] = x.to(DEV)
        ref[b].push(np.zeros((window, hq, d)), f64(old[0]), f64(old[1]))
    u = rounded(dtype)
    for lengths in pushes:
        n = sum(lengths)
        q, k, v = normal(g, n, hq, d, dtype=dtype), normal(g, n, hkv, d, dtype=dtype), normal(g, n, hkv, d, dtype=dtype)
        starts = torch.tensor([r.p for r in ref], device=DEV)
        offsets = torch.tensor([0] + list(lengths)).cumsum(0)
        kw = dict(offsets=offsets.to(DEV), max_tokens=max(lengths)) if ragged else {}
        out = idf.window_attend(q.to(DEV), k.to(DEV), v.to(DEV), *rings, starts, window=window, sinks=sinks, scale=scale, **kw)
        for b in range(streams):
            s = slice(int(offsets[b]), int(offsets[b + 1]))
            want, size, score = ref[b].push(f64(q[s]), f64(k[s]), f64(v[s]))
            keys = min(ref[b].p, window + sinks)
            bound = half_step(dtype) * np.abs(want) + (u + 2 * (2 * (d + 8) * W * score[..., None] + (keys + 16) * W)) * size
            within(out[s], want, bound, f"stream {b} of {lengths} from {ref[b].p - lengths[b]}")
    return rings, ref


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("hq,hkv,d,window,sinks", [(1, 1, 64, 1, 0), (4, 2, 64, 7, 2), (8, 1, 128, 64, 0), (3, 3, 80, 33, 5), (6, 2, 96, 100, 1), (2, 2, 16, 130, 64), (2, 1, 256, 40, 3),
                                                   (32, 2, 64, 20, 4)])
def test_window_single_tokens(dtype, hq, hkv, d, window, sinks):
    """From the first token on, past the point where the ring wraps."""
    pushes = [[1, 1, 1]] * 5 + [[60, 90, 1]] + [[1, 1, 1]] * 3 + [[64, 130, 31]] + [[1, 1, 1]] * 2
    window_streams(dtype, hq, hkv, d, window, sinks, 0, pushes, seed=window)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("room", [0, 9])
@pytest.mark.parametrize("hq,hkv,d,window,sinks", [(1, 1, 64, 1, 1), (4, 1, 64, 16, 0), (4, 4, 128, 65, 3), (10, 2, 80, 200, 70), (3, 1, 48, 31, 100), (2, 1, 256, 50, 2)])
def test_window_segments(dtype, hq, hkv, d, window, sinks, room):
    """Uneven segments, empty ones, ones longer than the ring, few tokens at a time."""
    pushes = [[0, 5, 17, 1], [130, 2, 0, 300], [9, 9, 9, 9], [1, 257, 40, 3], [0, 0, 1, 0]]
    window_streams(dtype, hq, hkv, d, window, sinks, room, pushes, seed=window + d)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("hq,hkv,d,window,sinks", [(6, 2, 64, 33, 2), (2, 2, 128, 16, 0), (16, 1, 96, 70, 40), (7, 1, 32, 1, 1)])
def test_window_rings_with_room_for_segments(dtype, hq, hkv, d, window, sinks):
    """The attention itself writes the ring while it is read: heads that leave tokens on two tiles, first tokens, slots that wrap."""
    window_streams(dtype, hq, hkv, d, window, sinks, 199, [[5, 1, 0], [200, 43, 129], [1, 1, 1], [64, 200, 2], [128, 7, 200], [2, 1, 3]], seed=d)
    window_streams(dtype, hq, hkv, d, window, sinks, 3, [[4, 2, 1], [1, 4, 0], [4, 4, 4], [3, 3, 3]] * 3, seed=d + 1)


def test_window_single_rows_split_many_times():
    """Lists of keys in more parts than a wave has lanes; first tokens ahead of them."""
    g = torch.Generator().manual_seed(15)
    d, window, sinks, start = 64, 40000, 3, 100000
    for dtype in TYPES:
        q, k, v = (normal(g, 1, h, d, dtype=dtype) for h in (2, 1, 1))
        rings = [normal(g, 1, sinks + window, 1, d, dtype=dtype) for _ in range(2)]
        out = idf.window_attend(*(x.to(DEV) for x in (q, k, v, *rings)), torch.tensor([start], device=DEV), window=window, sinks=sinks)
        slot = sinks + (start - sinks) % window                        # it holds the one token that has left the window
        seen = [np.concatenate([np.delete(f64(r[0, :, 0]), slot, 0), f64(x[:, 0])]) for r, x in zip(rings, (k, v))]
        for h in range(2):
            s = seen[0] @ f64(q[0, h]) / 8
            w = np.exp(s - s.max())
            w /= w.sum()
            want, size, score = w @ seen[1], w @ np.abs(seen[1]), (np.abs(seen[0]) @ np.abs(f64(q[0, h]))).max() / 8
            within(out[0, h], want, half_step(dtype) * np.abs(want) + (rounded(dtype) + 4 * (d + 8) * W * score + 2 * (window + 19) * W) * size)


@pytest.mark.parametrize("d", [4, 12, 20, 60, 68, 100, 132, 252])
def test_window_odd_heads(d):
    """Float32 heads whose end lies inside a fragment of eight values: what lies behind it, here NaN, is not read."""
    g = torch.Generator().manual_seed(d)
    pushes = [[1, 1], [13, 2], [1, 1], [90, 200], [3, 1], [1, 1]]
    window_streams(torch.float32, 2, 1, d, 30, 2, 0, pushes, seed=d)
    for lengths in ((1, 1), (4, 3), (70, 9)):
        n = sum(lengths)
        q, k, v = (torch.full((n, h, d + 4), float("nan"), device=DEV)[:, :, :d].copy_(normal(g, n, h, d, dtype=torch.float32)) for h in (3, 1, 1))
        offsets = torch.tensor((0,) + lengths).cumsum(0)
        out = idf.window_attend(q, k, v, window=30, offsets=offsets.to(DEV), max_tokens=max(lengths))
        for at, m in zip(offsets.tolist(), lengths):
            want, size, score = oracle.Attention(30, 0, 1 / np.sqrt(d)).push(*(f64(x[at:at + m]) for x in (q, k, v)))
            within(out[at:at + m], want, W * np.abs(want) + (4 * (d + 8) * W * score[..., None] + 2 * 46 * W) * size)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_window_long(dtype):
    """Few rows on a long axis, and many of them."""
    window_streams(dtype, 8, 2, 64, 3000, 5, 0, [[700, 2000], [1500, 1500], [1, 1], [3, 2], [1, 20], [1, 1]], seed=11)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_window_equal_segments_without_offsets(dtype):
    window_streams(dtype, 4, 2, 64, 40, 2, 0, [[16, 16, 16]] * 5, seed=5, ragged=False)
    window_streams(dtype, 4, 2, 64, 40, 2, 0, [[1, 1, 1]] * 5, seed=6, ragged=False)


def test_window_without_rings_and_strided():
    """Segments that see themselves only, as views of one projection with heads first."""
    g = torch.Generator().manual_seed(8)
    for dtype in TYPES:
        for hq, hkv, lengths in ((4, 2, (100, 33, 0, 1)), (2, 2, (5,)), (8, 1, (1, 1, 1))):
            n = sum(lengths)
            packed = normal(g, hq + 2 * hkv, n + 3, 64, dtype=dtype).to(DEV).transpose(0, 1)[1:n + 1]
            q, k, v = packed.split([hq, hkv, hkv], 1)
            store = torch.full((n + 2, hq, 72), 7.0, dtype=dtype, device=DEV)
            out = store[1:n + 1, :, :64]
            idf.window_attend(q, k, v, window=30, sinks=3, offsets=torch.tensor((0,) + lengths).cumsum(0).to(DEV), max_tokens=max(lengths), out=out)
            at = 0
            for m in lengths:
                want, size, score = oracle.Attention(30, 3, 1 / 8).push(*(f64(x[at:at + m]) for x in (q, k, v)))
                within(out[at:at + m], want, half_step(dtype) * np.abs(want) + (rounded(dtype) + 4 * 72 * W * score[..., None] + 2 * 50 * W) * size)
                at += m
            assert torch.all(store[0] == 7) and torch.all(store[-1] == 7) and torch.all(store[:, :, 64:] == 7)


def test_window_far_positions_and_stream_ids():
    """Positions beyond 32 bits; rings picked by ids; ids and starts that are none leave their rows as they are."""
    window_streams(torch.bfloat16, 4, 2, 64, 50, 0, 3, [[40, 60], [1, 1], [70, 5], [1, 1]], seed=9, start=(1 << 40) + 12345)
    g = torch.Generator().manual_seed(10)
    q, k, v = (normal(g, 6, h, 64, dtype=torch.float32).to(DEV) for h in (2, 1, 1))
    rings = [normal(g, 5, 20, 1, 64, dtype=torch.float32).to(DEV) for _ in range(2)]
    before = [r.clone() for r in rings]
    ids = torch.tensor([3, -1, 5, 0, 1, 2], dtype=torch.int32, device=DEV)
    starts = torch.tensor([0, 0, 0, 17, -4, 100], device=DEV)
    out = torch.full_like(q, 9.0)
    idf.window_attend(q, k, v, *rings, starts, window=20, stream_ids=ids, out=out)
    assert torch.all(out[[1, 2, 4]] == 9) and torch.all(out[[0, 3, 5]] != 9)
    assert torch.allclose(out[0], v[0].expand(2, -1))                  # a first token sees itself
    for r, old, new in zip(rings, before, (k, v)):
        for i, ring, slot in ((0, 3, 0), (3, 0, 17), (5, 2, 0)):
            assert torch.equal(r[ring, slot], new[i])
            old[ring, slot] = new[i]
        assert torch.equal(r, old)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("m", [4, 200])
def test_window_offsets_that_lie(dtype, m):
    """Offsets beyond the tokens, in falling order or with segments longer than max_tokens stay inside."""
    g = torch.Generator().manual_seed(12)
    n = 3 * m
    q, k, v = (normal(g, n, h, 64, dtype=dtype).to(DEV) for h in (2, 1, 1))
    out = torch.full((n + 8, 2, 64), 9.0, dtype=dtype, device=DEV)
    offsets = torch.tensor([-5, m, 2 * m + 5, 2 * m, 1 << 40], device=DEV)
    idf.window_attend(q, k, v, window=1000, offsets=offsets, max_tokens=m, out=out[:n])
    want = idf.window_attend(q[:m], k[:m], v[:m], window=1000)
    assert torch.equal(out[:m], want) and torch.all(out[n:] == 9)
    assert torch.all(out[2 * m:2 * m] != 9) and torch.all(out[2 * m:] [:m] != 9)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("n,hq", [(1, 2), (3, 2), (40, 4), (300, 2)])
def test_window_what_is_not_seen_does_not_count(dtype, bad, n, hq):
    """Infinities and NaN in keys and values that a query does not see, in those of later tokens too, leave its output as it is."""
    g = torch.Generator().manual_seed(n)
    q, k, v = (normal(g, n, h, 64, dtype=dtype) for h in (hq, 2, 2))
    rings = [normal(g, 1, 33, 2, 64, dtype=dtype) for _ in range(2)]
    starts = torch.tensor([100], device=DEV)

    def go(k, v, rings):
        rings = [r.to(DEV) for r in rings]
        return idf.window_attend(q.to(DEV), k.to(DEV), v.to(DEV), *rings, starts, window=20, sinks=2)
    want = go(k, v, rings)
    # the ring has room for 31 tokens behind the first two, the newest 19 of which are seen by the first query
    hidden = [r.clone() for r in rings]
    for p in range(100 - 31, 100 - 19):
        for r in hidden:
            r[0, 2 + (p - 2) % 31] = bad
    assert torch.equal(go(k, v, hidden), want)
    if n > 2:
        for x in (0, 1):
            later = [k.clone(), v.clone()]
            later[x][n // 2] = bad
            got = go(*later, rings)
            near = torch.zeros(n, dtype=torch.bool)
            near[n // 2:n // 2 + 20] = True
            # rows apart from those that see the token: the same but for the order in which a fallback adds
            a, b = got[~near].float(), want[~near].float()
            assert torch.allclose(a, b, rtol=4 * half_step(dtype), atol=(2 * half_step(dtype) if dtype != torch.float32 else 1e-6) * float(v.float().abs().max())), x
            if x == 1:
                assert not torch.isfinite(got[near].float()).any()


def test_window_large_scores():
    """Scores far apart: weights of one and of zero, no overflow."""
    g = torch.Generator().manual_seed(14)
    for dtype in TYPES:
        q, k, v = (normal(g, 90, 2, 64, dtype=dtype) for _ in range(3))
        q = (q.float() * 100).to(dtype)
        out = idf.window_attend(q.to(DEV), k.to(DEV), v.to(DEV), window=50)
        want, size, score = oracle.Attention(50, 0, 1 / 8).push(f64(q), f64(k), f64(v))
        within(out, want, half_step(dtype) * np.abs(want) + (rounded(dtype) + 4 * 72 * W * score[..., None] + 2 * 66 * W) * size)


# ---- linear attention with a decay ----

def decay_case(dtype, hq, hkv, dk, dv, lengths, seed=0, with_state=True, ragged=True, in_place=False, log_decay=None, state_scale=1.0):
    g = torch.Generator().manual_seed(seed)
    n, streams = sum(lengths), len(lengths)
    q, k, v = normal(g, n, hq, dk, dtype=dtype), normal(g, n, hkv, dk, dtype=dtype), normal(g, n, hkv, dv, dtype=dtype)
    log_decay = -torch.rand(hkv, generator=g) * torch.tensor([1.0, 0.1, 0.01, 0.001])[torch.arange(hkv) % 4] if log_decay is None else log_decay
    state = state_scale * torch.randn(streams, hkv, dk, dv, generator=g)
    s_in = state.to(DEV) if with_state else None
    s_out = s_in if in_place else torch.full(state.shape, float("nan"), device=DEV)
    offsets = torch.tensor([0] + list(lengths)).cumsum(0)
    kw = dict(offsets=offsets.to(DEV), max_tokens=max(lengths)) if ragged else {}
    out = idf.decay_attend(q.to(DEV), k.to(DEV), v.to(DEV), log_decay.to(DEV), s_in, s_out, **kw)
    u, scale = rounded(dtype), 1 / np.sqrt(dk)
    for b in range(streams):
        s = slice(int(offsets[b]), int(offsets[b + 1]))
        want, size, end, end_size = oracle.decay(f64(q[s]), f64(k[s]), f64(v[s]), f64(log_decay), f64(state[b]) if with_state else np.zeros(state.shape[1:]), scale)
        m = lengths[b]
        powers = np.abs(f64(log_decay)).clip(max=1e4) * 1.0
        # a power of the decay that still counts has an exponent of at most 100 (e^-100 is nothing next to 2^-24)
        powers = np.minimum(powers * max(m, 1), 100.0)
        steps = 2 * (m + 16 + powers) * W
        within(out[s], want, half_step(dtype) * np.abs(want) + (2 * u + steps.repeat(hq // hkv)[None, :, None] + 2 * dk * W) * size, f"segment {b} of {lengths}: out")
        within(s_out[b], end, steps[:, None, None] * end_size + 1e-30, f"segment {b} of {lengths}: state")


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("hq,hkv,dk,dv", [(1, 1, 64, 64), (4, 2, 128, 128), (3, 3, 32, 80), (2, 1, 96, 64), (8, 1, 64, 200), (1, 1, 256, 32), (2, 2, 8, 8), (4, 4, 128, 64)])
@pytest.mark.parametrize("lengths", [(1, 1, 1), (1, 0, 1), (2, 5, 16, 3), (63, 64, 65, 0, 1), (130, 17)])
def test_decay(dtype, hq, hkv, dk, dv, lengths):
    decay_case(dtype, hq, hkv, dk, dv, lengths, seed=dk + len(lengths))


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("hq,hkv,dk,dv", [(2, 1, 64, 64), (2, 2, 128, 80), (1, 1, 200, 64)])
@pytest.mark.parametrize("lengths", [(2, 1, 0), (4, 3, 2), (12, 0, 7), (13, 1, 5)])
def test_decay_few_tokens(dtype, hq, hkv, dk, dv, lengths):
    """Both sides of the line between tokens one by one and chunks."""
    decay_case(dtype, hq, hkv, dk, dv, lengths, seed=sum(lengths))


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("with_state,in_place", [(False, False), (True, True)])
def test_decay_states(dtype, with_state, in_place):
    for lengths in ((1, 1), (9, 9), (200, 200)):
        decay_case(dtype, 2, 2, 64, 64, lengths, seed=1, with_state=with_state, in_place=in_place, ragged=False)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_decay_long(dtype):
    """Long enough to be split over the time axis, beside short ones."""
    decay_case(dtype, 2, 1, 64, 96, (3000, 1, 0, 700), seed=2)
    decay_case(dtype, 1, 1, 128, 128, (4097,), seed=3, in_place=True)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_decay_extremes(dtype):
    """No decay at all, and one that leaves nothing (log of zero)."""
    for lengths in ((1, 3), (150, 70)):
        decay_case(dtype, 3, 3, 64, 64, lengths, seed=4, log_decay=torch.tensor([0.0, -float("inf"), -200.0]))


def test_decay_strided_ids_and_no_state_out():
    g = torch.Generator().manual_seed(5)
    for dtype in TYPES:
        for m in (1, 6, 100):
            packed = normal(g, 3 * m, 4 + 2 + 2, 64, dtype=dtype).to(DEV)
            q, k, v = packed.split([4, 2, 2], 1)
            state = torch.randn(4, 2, 64, 64, generator=g).to(DEV)
            before = state.clone()
            ids = torch.tensor([2, 7, 0], dtype=torch.int32, device=DEV)
            log_decay = torch.tensor([-0.1, -0.01], device=DEV)
            out = torch.full((3 * m, 4, 64), 9.0, dtype=dtype, device=DEV)
            none = idf.decay_attend(q, k, v, log_decay, state, stream_ids=ids)
            idf.decay_attend(q, k, v, log_decay, state, state, stream_ids=ids, out=out)
            assert torch.equal(state[[1, 3]], before[[1, 3]]) and torch.all(out[m:2 * m] == 9)
            for s, ring in ((0, 2), (2, 0)):
                one = before[ring:ring + 1].clone()
                rows = slice(s * m, (s + 1) * m)
                want = idf.decay_attend(q[rows], k[rows], v[rows], log_decay, one, one)
                assert torch.equal(out[rows], want) and torch.equal(none[rows], want) and torch.equal(state[ring], one[0])


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_decay_later_tokens_do_not_count(dtype, bad):
    g = torch.Generator().manual_seed(6)
    for n in (3, 100):
        q, k, v = (normal(g, n, 1, 64, dtype=dtype) for _ in range(3))
        log_decay = torch.tensor([-0.05], device=DEV)
        go = lambda k, v: idf.decay_attend(q.to(DEV), k.to(DEV), v.to(DEV), log_decay)      # noqa: E731
        want = go(k, v)
        for x in (0, 1):
            later = [k.clone(), v.clone()]
            later[x][n // 2] = bad
            got = go(*later)
            a, b = got[:n // 2].float(), want[:n // 2].float()
            assert torch.allclose(a, b, rtol=4 * half_step(dtype), atol=4 * half_step(dtype) * float(b.abs().max()))
            assert not torch.isfinite(got[n // 2:].float()).any()


# ---- streams and graphs ----

def test_another_stream_and_a_graph():
    """The calls go where torch's current stream is, and a recorded step follows positions that are counted on the device."""
    g = torch.Generator().manual_seed(20)
    B, hq, hkv, d, window = 3, 4, 2, 64, 24
    rings = [torch.zeros(B, window, hkv, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    state = torch.zeros(B, hkv, d, d, device=DEV)
    log_decay = torch.tensor([-0.1, -0.02], device=DEV)
    f, amplitude = idf.rotary_frequencies(d, device=DEV)
    w = torch.ones(d, device=DEV)
    xs = [normal(g, B, hq + 2 * hkv, d, dtype=torch.bfloat16).to(DEV) for _ in range(40)]

    def step(x, positions, rings, state):
        q, k, v = x.split([hq, hkv, hkv], 1)
        q, k = idf.norm_rotate(q, k, positions, f, amplitude=amplitude, q_weight=w, k_weight=w)
        a = idf.window_attend(q, k, v, *rings, positions, window=window)
        b = idf.decay_attend(q, k, v, log_decay, state, state)
        return a, b
    want, p, r, s = [], torch.zeros(B, dtype=torch.int64, device=DEV), [x.clone() for x in rings], state.clone()
    for x in xs:
        a, b = step(x, p, r, s)
        want.append((a.clone(), b.clone()))
        p += 1
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    x0, p = xs[0].clone(), torch.zeros(B, dtype=torch.int64, device=DEV)
    with torch.cuda.stream(side):
        step(x0, p, [x.clone() for x in rings], state.clone())
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = step(x0, p, rings, state)
        p += 1
    for x, (wa, wb) in zip(xs, want):
        x0.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, wa) and torch.equal(b, wb)


def test_same_bits_every_time():
    g = torch.Generator().manual_seed(21)
    for n, window in ((1, 5000), (300, 200)):
        q, k, v = (normal(g, 2 * n, h, 64, dtype=torch.bfloat16).to(DEV) for h in (4, 1, 1))
        rings = [normal(g, 2, window + n, 1, 64, dtype=torch.bfloat16).to(DEV) for _ in range(2)]
        starts = torch.tensor([20000, 4000], device=DEV)
        a = [idf.window_attend(q, k, v, *rings, starts, window=window) for _ in range(3)]
        assert torch.equal(a[0], a[1]) and torch.equal(a[0], a[2])
    q, k, v = (normal(g, 4000, 1, 64, dtype=torch.bfloat16).to(DEV) for _ in range(3))
    a = [idf.decay_attend(q, k, v, torch.tensor([-0.01], device=DEV)) for _ in range(3)]
    assert torch.equal(a[0], a[1]) and torch.equal(a[0], a[2])


# ---- the two ways into the library ----

def test_both_ways_into_the_library_agree(monkeypatch):
    """Compiled code takes plain tensors; what it leaves goes by ctypes, with the same results and outputs where they were asked for."""
    from paper_1804_10727_amd import tokens
    g = torch.Generator().manual_seed(30)
    q, k, v = (normal(g, 6, h, 64, dtype=torch.bfloat16).to(DEV) for h in (4, 2, 2))
    rings = [normal(g, 3, 12, 2, 64, dtype=torch.bfloat16).to(DEV) for _ in range(2)]
    starts = torch.tensor([30, 4, 0], device=DEV)
    positions = torch.arange(6, device=DEV)
    f, _ = idf.rotary_frequencies(64, device=DEV)
    w = torch.rand(64, generator=g).to(DEV)
    state = torch.randn(3, 2, 64, 64, generator=g).to(DEV)
    log_decay = torch.tensor([-0.1, -0.2], device=DEV)
    offsets = torch.tensor([0, 3, 4, 6], device=DEV)
    ids = torch.tensor([2, 0, 1], dtype=torch.int32, device=DEV)

    def everything():
        r, s = [x.clone() for x in rings], state.clone()
        into = torch.zeros_like(q)
        got = [*idf.norm_rotate(q, k, positions, f, q_weight=w), *idf.norm_rotate(q, k, positions, f, layout="interleaved", amplitude=2, q_out=into),
               idf.window_attend(q, k, v, *r, starts, window=10, sinks=2), idf.window_attend(q, k, v, *r, starts, window=10, sinks=1, offsets=offsets, max_tokens=3),
               idf.window_attend(q, k, v, window=4, scale=1), idf.window_attend(q[:3], k[:3], v[:3], *r, starts, window=12, stream_ids=ids, out=into[:3]),
               idf.decay_attend(q, k, v, log_decay, s, s), idf.decay_attend(q, k, v, log_decay, offsets=offsets, max_tokens=3),
               idf.decay_attend(q, k, v, log_decay, n_segments=2), idf.decay_attend(q, k, v, log_decay, s, None, stream_ids=ids)]
        return got + [into, *r, s]
    want = everything()
    called = []
    real = tokens._direct
    monkeypatch.setattr(tokens, "_direct", lambda name, *a: called.append((name, real(name, *a) is not None)))
    got = everything()
    assert len(called) == 10 and all(taken for _, taken in called)
    # (each call ran both ways here: what is updated in place went twice, so only what is not is compared)
    for i in (0, 1, 2, 3, 6, 9, 10):
        assert torch.equal(got[i], want[i]), i
    monkeypatch.setattr(tokens, "_direct", lambda *a: None)
    for a, b in zip(everything(), want):
        assert torch.equal(a, b)


def test_python_refuses_on_the_gpu():
    q = torch.zeros(4, 2, 64, device=DEV)
    f, _ = idf.rotary_frequencies(64, device=DEV)
    ring = torch.zeros(2, 8, 2, 64, device=DEV)
    p = torch.zeros(4, dtype=torch.int64, device=DEV)
    for call in (lambda: idf.norm_rotate(q, q, p[:3], f), lambda: idf.norm_rotate(q, q, p.int(), f), lambda: idf.norm_rotate(q, q, p, f.float()),
                 lambda: idf.norm_rotate(q, q[:3], p, f), lambda: idf.norm_rotate(q, q, p, f, q_weight=f), lambda: idf.norm_rotate(q, q, p, f, q_out=q[:3]),
                 lambda: idf.norm_rotate(q, q.cpu(), p, f), lambda: idf.norm_rotate(q, q, p.cpu(), f),
                 lambda: idf.window_attend(q, q, q[:3], window=4), lambda: idf.window_attend(q, q, q, ring, window=4), lambda: idf.window_attend(q, q, q, ring, ring[:1], window=4),
                 lambda: idf.window_attend(q, q, q, ring.bfloat16(), ring.bfloat16(), window=4), lambda: idf.window_attend(q, q, q, window=4, offsets=p),
                 lambda: idf.window_attend(q, q, q, ring[:, ::2], ring[:, ::2], window=4), lambda: idf.window_attend(q, q, q, window=4, starts=p[:3]),
                 lambda: idf.window_attend(q, q, q, window=4, out=q[:, :, ::2]), lambda: idf.decay_attend(q, q, q, p), lambda: idf.decay_attend(q, q, q, p.float()),
                 lambda: idf.decay_attend(q, q, q, p[:2].float(), torch.zeros(1, 2, 64, 32, device=DEV)), lambda: idf.decay_attend(q, q, q, p[:2].float(), n_segments=3),
                 lambda: idf.decay_attend(q, q, q, p[:2].float(), torch.zeros(1, 2, 64, 64, device=DEV), torch.zeros(2, 2, 64, 64, device=DEV))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: idf.norm_rotate(q.half(), q.half(), p, f), lambda: idf.window_attend(q, q, q, window=0), lambda: idf.window_attend(q, q, q, ring, ring, window=9),
                 lambda: idf.window_attend(q, q, q, window=4, scale=-1.0), lambda: idf.decay_attend(q, q, q, p[:2].float(), scale=float("nan"))):
        with pytest.raises(idf.IdfError):
            call()
