"""The operators that mix the tokens of a stream, from their definitions: numpy, float64, token by token, whole histories kept.

Every function returns what is asked for and, beside it, the sums of absolute terms that a tolerance is derived from.
"""
from __future__ import annotations

import numpy as np


def norm_rotate(x, positions, frequencies, interleaved, amplitude, weight, eps):
    """x [n][heads][d], one weight [d] or None: normalised and turned.  (values, absolute terms)."""
    x = np.array(x, dtype=np.float64)
    if weight is not None:
        x = np.asarray(weight, np.float64) * x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    y, size = x.copy(), np.abs(x)
    r = 2 * len(frequencies)
    for i, f in enumerate(frequencies):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
        # the angle as an exact product taken to turns, so that far positions lose nothing
        angle = np.array([float(np.fmod(np.longdouble(p) * np.longdouble(f), 2 * np.longdouble(np.pi))) for p in positions])[:, None]
        c, s = amplitude * np.cos(angle), amplitude * np.sin(angle)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        size[..., a], size[..., b] = np.abs(x[..., a] * c) + np.abs(x[..., b] * s), np.abs(x[..., b] * c) + np.abs(x[..., a] * s)
    return y, size


def visible(p, window, sinks):
    """Positions that the token at position p attends to."""
    return [j for j in range(p + 1) if j > p - window or j < sinks]


class Attention:
    """One stream: the keys and values of every position, kept for good."""

    def __init__(self, window, sinks, scale, start=0):
        self.window, self.sinks, self.scale, self.p, self.first = window, sinks, scale, start, start
        self.k = self.v = None

    def push(self, q, k, v):
        """q [n][hq][d], k, v [n][hkv][d]: (out, attention of the absolute values, largest absolute terms of a score)."""
        q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
        group = q.shape[1] // k.shape[1]
        out, size, score = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
        self.k, self.v = (new if old is None else np.concatenate([old, new]) for old, new in ((self.k, k), (self.v, v)))
        for t in range(q.shape[0]):
            low = max(self.first, self.p - self.window + 1)
            js = list(range(self.first, min(self.sinks, low))) + list(range(low, self.p + 1))
            kk, vv = self.k[np.array(js) - self.first], self.v[np.array(js) - self.first]
            for h in range(q.shape[1]):
                s = self.scale * (kk[:, h // group] @ q[t, h])
                w = np.exp(s - s.max())
                w /= w.sum()
                out[t, h] = w @ vv[:, h // group]
                size[t, h] = w @ np.abs(vv[:, h // group])
                score[t, h] = self.scale * (np.abs(kk[:, h // group]) @ np.abs(q[t, h])).max()
            self.p += 1
        return out, size, score


def decay(q, k, v, log_decay, state, scale):
    """q [n][hq][dk], k [n][hkv][dk], v [n][hkv][dv], state [hkv][dk][dv]: (out, its absolute terms, state, its absolute terms)."""
    q, k, v, log_decay = (np.asarray(x, np.float64) for x in (q, k, v, log_decay))
    group = q.shape[1] // k.shape[1]
    s = np.array(state, dtype=np.float64)
    size = np.abs(s)
    out = np.zeros(q.shape[:2] + (v.shape[2],))
    out_size = np.zeros_like(out)
    lam = np.exp(log_decay)[:, None, None]
    for t in range(q.shape[0]):
        kv = k[t][:, :, None] * v[t][:, None, :]
        s, size = lam * s + kv, lam * size + np.abs(kv)
        for h in range(q.shape[1]):
            out[t, h] = scale * (q[t, h] @ s[h // group])
            out_size[t, h] = scale * (np.abs(q[t, h]) @ size[h // group])
    return out, out_size, s, size
