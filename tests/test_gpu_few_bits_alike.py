"""The same by other ways: attention over 4-bit rings against the window's attention over the values that they stand for, and a stream through the mixer in other cuts."""
import numpy as np
import pytest
import torch

import paper_1804_10727_amd as idf
from oracle import few_bits as oracle
from paper_1804_10727_amd import mixing
from paper_1804_10727_amd.mixing import FewBitsMixer
from test_gpu_nibble import alike, f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
W = 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("tokens", [1, 7, 40, 700])
def test_the_windows_attention_over_the_rings_values(tokens, dim, dtype):
    """Hundreds of keys and first tokens to a query, from the tokens before a segment and its own: single tokens, few rows, tiles of rows."""
    g = torch.Generator().manual_seed(tokens + dim)
    streams, hq, hkv, window, sinks, have = 2, 4, 2, 300, 5, 500
    q, k, v = (torch.randn(streams, have + tokens, h, dim, generator=g).to(dtype).to(DEV) for h in (hq, hkv, hkv))
    ring = idf.nibble_ring(streams, have + tokens, hkv, dim, DEV)         # (no slot is used twice: the values of all tokens can be had)
    idf.nibble_append(k.flatten(0, 1), v.flatten(0, 1), ring, sinks=sinks)
    kk, vv = idf.nibble_values(ring, dtype)
    starts = torch.full((streams,), have, device=DEV)
    mine = q[:, have:].flatten(0, 1)
    got = idf.nibble_attend(mine, ring, starts, window=window, sinks=sinks)
    # the window's: keys of the segment by themselves, those before them from a ring
    old = [torch.zeros(streams, sinks + window, hkv, dim, dtype=dtype, device=DEV) for _ in range(2)]
    idf.window_attend(q[:, :have].flatten(0, 1), kk[:, :have].flatten(0, 1), vv[:, :have].flatten(0, 1), *old, torch.zeros_like(starts), window=window, sinks=sinks)
    want = idf.window_attend(mine, kk[:, have:].flatten(0, 1), vv[:, have:].flatten(0, 1), *old, starts, window=window, sinks=sinks)
    assert alike(got, want, dtype, vv)
    # and it is no other window, no other scale and no other key that gives the same
    for other in (dict(window=window - 40, sinks=sinks), dict(window=window, sinks=0), dict(window=window, sinks=sinks, scale=0.5 * dim ** -0.5)):
        assert not alike(idf.nibble_attend(mine, ring, starts, **other), want, dtype, vv)


def test_cuts_of_a_stream(monkeypatch):
    """Rows pushed one by one, in pieces, in uneven ones: in every cut what the layers' definitions give for the whole stream, and rings that hold the same blocks to the bit.  Products
    are taken in float64 here, from the same 8-bit weights, so that no code of a row goes the other way by the order of an earlier sum."""
    def product(x, weight, scales, bias=None):
        y = x.double() @ (weight.double() * scales.double()[:, None]).T[:x.shape[1]]
        return (y if bias is None else y + bias.double()).float()
    monkeypatch.setattr(mixing, "project_rows", product)
    g = torch.Generator().manual_seed(7)
    streams, n, channels, heads, kv, dim, window, sinks = 3, 60, 48, 4, 2, 64, 20, 3
    rows = torch.randn(streams, n, channels, generator=g).to(DEV)
    outs, rings, states = [], [], []
    for cut in (1, 4, 9, None):
        m = FewBitsMixer(channels, streams, heads=heads, kv_heads=kv, dim=dim, window=window, sinks=sinks, room=17)
        at, got, turn = [0] * streams, [[] for _ in range(streams)], 0
        while min(at) < n:
            counts = [min(n - a, cut if cut else (turn * 5 + b * 7) % 18) for b, a in enumerate(at)]
            turn += 1
            y = m.push(torch.cat([rows[b, a:a + c] for b, (a, c) in enumerate(zip(at, counts))]), None if cut and turn % 2 else counts)
            for b, part in enumerate(y.split(counts)):
                got[b].append(part)
                at[b] += counts[b]
        assert m.starts.tolist() == [n] * streams
        outs.append(torch.stack([torch.cat(p) for p in got]))
        rings.append([t[:, :, [p if p < sinks else sinks + (p - sinks) % (t.shape[2] - sinks) for p in [*range(sinks), *range(n - window, n)]]] for t in m.rings])
        states.append(m.state)
    assert all(torch.equal(a, b) for other in rings[1:] for a, b in zip(rings[0], other))
    # the whole stream: what every token puts into a ring that has room for all, and queries, then in float64 with the error of each step carried on
    packed = product(rows.flatten(0, 1), *m.weights[0]).unflatten(1, (-1, dim))
    q, k, v = packed.split([heads, kv, kv], 1)
    positions = torch.arange(n, device=DEV).repeat(streams)
    q, _ = idf.norm_rotate(q, k[:, :0], positions, m.frequencies, amplitude=m.amplitude, q_weight=m.q_weight)
    ring = idf.nibble_ring(streams, n, kv, dim, DEV)
    idf.nibble_append(k, v, ring, frequencies=m.frequencies, amplitude=m.amplitude, k_weight=m.k_weight)
    keys, values = (t.double().cpu().numpy() for t in idf.nibble_values(ring, torch.float32))
    weights = [f64(w).astype(np.float64)[:, :c] * f64(s)[:, None] for (w, s), c in zip(m.weights, (channels, heads * dim, channels))]
    q, bias = f64(q).reshape(streams, n, heads, dim), f64(m.gate_bias)
    for b in range(streams):
        h, off = np.zeros(channels), np.zeros(channels)
        wants, bounds = [], []
        for t in range(n):
            js = [j for j in range(t + 1) if j > t - window or j < sinks]
            seen, error = np.zeros((heads, dim)), np.zeros((heads, dim))
            for i in range(heads):
                kk, vv = keys[b, js, i * kv // heads], values[b, js, i * kv // heads]
                s = kk @ q[b, t, i] / np.sqrt(dim)
                w = np.exp(s - s.max())
                w /= w.sum()
                score = (np.abs(kk) @ np.abs(q[b, t, i])).max() / np.sqrt(dim)
                seen[i] = w @ vv
                error[i] = W * np.abs(seen[i]) + 2 * (2 * (dim + 8) * W * score + (len(js) + 16) * W) * (w @ np.abs(vv))
            x = f64(rows[b, t])
            one = x + weights[1] @ seen.ravel()
            e = np.abs(weights[1]) @ error.ravel() + 3 * W * (np.abs(x) + np.abs(weights[1] @ seen.ravel()))
            both = weights[2] @ one + bias
            eb = np.abs(weights[2]) @ e + 2 * W * np.abs(both)
            gate, new = both[:channels], both[channels:]
            keep, take = oracle.sigmoid(gate)
            # a state moves with what comes in, and by a (1 - a) (h - x) with its gate; a step's own roundings as the oracle of the recurrence has them
            off = keep * off + take * eb[channels:] + keep * take * np.abs(h - new) * eb[:channels] + W * (12 + 3 * np.abs(gate)) * (take * np.abs(new) + np.abs(h))
            h = keep * h + take * new
            wants.append(one + h)
            bounds.append(1.1 * (e + off) + W * np.abs(one + h))     # (a tenth more than the first order)
        wants, bounds = np.array(wants), np.array(bounds)
        assert np.median(bounds) < 0.02 * wants.std()                 # (or they would say nothing)
        for o, s in zip(outs, states):
            assert np.all(np.abs(f64(o[b]) - wants) <= bounds) and np.all(np.abs(f64(s[b]) - h) <= 1.1 * off + W * np.abs(h))
