"""Layers in few bits and the gated recurrence, from their definitions: numpy, float64, value by value or token by token.

Every function of real numbers returns, beside what is asked for, the sums of absolute terms that a tolerance is derived from.
"""
from __future__ import annotations

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32
GATE = 87.0


def quantize_rows(x):
    """(codes, scales) of the rows of x; a row with a value that is not finite: zeros and NaN."""
    x = np.asarray(x, np.float64)
    most = np.abs(x).max(axis=1)
    fine = np.isfinite(most)
    codes = np.zeros(x.shape, np.int64)
    some = fine & (most > 0)
    codes[some] = np.rint(127 * x[some] / most[some, None]).astype(np.int64)
    return codes, np.where(fine, most / 127, np.nan)


def blocks(y):
    """y [.., dim]: (codes [.., dim] of 0 .. 15, powers [.., dim / 32] as bytes).  The nearest level by the borders between them, halfway to the even
    code."""
    y = np.asarray(y, np.float64)
    y = y.reshape(y.shape[:-1] + (y.shape[-1] // BLOCK, BLOCK))
    most = np.abs(y).max(axis=-1)
    fine = np.isfinite(most)
    e = np.full(most.shape, -100)
    for power in range(-100, 125):
        e = np.where(most > 7 * 2.0 ** power, power + 1, e)
    with np.errstate(invalid="ignore"):
        size = np.abs(y) * 2.0 ** -e[..., None].astype(np.float64)
    code = np.zeros(y.shape, np.int64)
    for i in range(7):
        border = (LEVELS[i] + LEVELS[i + 1]) / 2
        code += (size >= border) if i % 2 else (size > border)
    code |= np.signbit(y).astype(np.int64) << 3
    code = np.where(fine[..., None], code, 0)
    return code.reshape(code.shape[:-2] + (code.shape[-2] * BLOCK,)), np.where(fine, e + 127, 255).astype(np.uint8)


def block_values(codes, powers):
    """What codes 0 .. 15 and powers stand for."""
    v = np.where(codes & 8, -1.0, 1.0) * LEVELS[codes & 7]
    p = np.where(powers == 255, np.nan, 2.0 ** (powers.astype(np.float64) - 127))
    return v * np.repeat(p, BLOCK, axis=-1)


def unpacked(codes):
    """Codes two to a byte, the even one in the low bits, as they lie in a ring."""
    codes = np.asarray(codes)
    return np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (2 * codes.shape[-1],)).astype(np.int64)


def sigmoid(g):
    g = np.where(np.isnan(g), g, np.clip(g, -GATE, GATE))
    return 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))


def gate_scan(x, g, state):
    """x, g [n][channels], state [channels]: (h of every token, their absolute terms, their errors in units of float32's half steps)."""
    x, g = np.asarray(x, np.float64), np.asarray(g, np.float64)
    keep, take = sigmoid(g)
    h, size, error = np.asarray(state, np.float64).copy(), np.abs(np.asarray(state, np.float64)), np.zeros(x.shape[1])
    hs, sizes, errors = (np.empty(x.shape) for _ in range(3))
    for t in range(len(x)):
        h, size = keep[t] * h + take[t] * x[t], keep[t] * size + take[t] * np.abs(x[t])
        # a gate is off by some ten roundings and by those of its exponent; the step by a few of the terms
        error = keep[t] * error + (12 + 3 * np.abs(np.clip(g[t], -GATE, GATE))) * (take[t] * np.abs(x[t]) + size)
        hs[t], sizes[t], errors[t] = h, size, error
    return hs, sizes, errors


def gate_scan_backward(x, g, state, grad_out, grad_end):
    """(grad_x, grad_gates, grad_state) and of each its error in units of float32's half steps."""
    x, g, d = (np.asarray(v, np.float64) for v in (x, g, grad_out))
    keep, take = sigmoid(g)
    hs, sizes, errors = gate_scan(x, g, state)
    first = np.asarray(state, np.float64)[None]
    was, was_size, was_error = np.concatenate([first, hs])[:-1], np.concatenate([np.abs(first), sizes])[:-1], np.concatenate([0 * first, errors])[:-1]
    flow, size, error = np.asarray(grad_end, np.float64).copy(), np.abs(np.asarray(grad_end, np.float64)), np.zeros(x.shape[1])
    grads, bounds = [np.empty(x.shape) for _ in range(2)], [np.empty(x.shape) for _ in range(2)]
    for t in reversed(range(len(x))):
        off = 12 + 3 * np.abs(np.clip(g[t], -GATE, GATE))
        slope = keep[t] * take[t]
        now, now_size, now_error = d[t] + flow, np.abs(d[t]) + size, error + np.abs(d[t]) + size
        grads[0][t], bounds[0][t] = take[t] * now, take[t] * (now_error + off * now_size)
        apart, apart_size = was[t] - x[t], was_size[t] + np.abs(x[t])
        grads[1][t] = now * apart * slope
        bounds[1][t] = slope * (now_error * apart_size + now_size * (was_error[t] + (2 * off + 4) * apart_size))
        flow, size = keep[t] * now, keep[t] * now_size
        error = keep[t] * (now_error + off * now_size)
    return grads[0], grads[1], flow, bounds[0], bounds[1], error
