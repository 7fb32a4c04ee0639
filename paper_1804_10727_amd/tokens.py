"""The operators that mix the tokens of streams (include/idf.h, last sections) on torch tensors: argument marshalling only.

Everything is enqueued on the current stream of the tensors' device.  There is no backward pass but that of gate_scan_recorded: tensors that require
gradients are refused elsewhere where gradients are recorded, taken under torch.no_grad(); tensors that carry a tangent of torch's forward mode are
refused everywhere.  Packed tokens [token][head][value]; a tensor whose values lie apart, or whose rows do not begin at multiples of 16 bytes where the
library asks for that, is copied first.  Rows of a result that no segment has are left as they are, where a call makes the result itself as its memory
was (but for the recurrence's: zeros).
"""
from __future__ import annotations

import ctypes as C
import math
from typing import NamedTuple

import numpy as np

from .binding import _check, load_library, load_tokens

_PREC = {}
_native = None               # csrc/tokens.cpp
_current_stream = None
SCALING = {None: 0, "linear": 1, "base": 2, "parts": 3}


class _Tokens(C.Structure):
    _fields_ = [("base", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class _NormRotate(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("precision", "heads_q", "heads_k", "head_dim", "rotary_dim", "interleaved")] +
                [("n_tokens", C.c_int64)] + [(n, _Tokens) for n in ("q", "k", "q_out", "k_out")] +
                [(n, C.c_void_p) for n in ("positions", "frequencies", "q_weight", "k_weight")] +
                [("amplitude", C.c_double), ("eps", C.c_float)])


class _Window(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("precision", "heads_q", "heads_kv", "head_dim")] +
                [("n_tokens", C.c_int64), ("max_tokens", C.c_int64), ("n_segments", C.c_int), ("n_streams", C.c_int),
                 ("slots", C.c_int64), ("window", C.c_int), ("sinks", C.c_int), ("scale", C.c_float)] +
                [(n, _Tokens) for n in ("q", "k", "v", "out")] +
                [(n, C.c_void_p) for n in ("k_ring", "v_ring", "offsets", "starts", "stream_ids", "workspace")] +
                [("workspace_bytes", C.c_size_t)])


class _Decay(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("precision", "heads_q", "heads_kv", "dim_k", "dim_v")] +
                [("n_tokens", C.c_int64), ("max_tokens", C.c_int64), ("n_segments", C.c_int), ("n_streams", C.c_int), ("scale", C.c_float)] +
                [(n, _Tokens) for n in ("q", "k", "v", "out")] +
                [(n, C.c_void_p) for n in ("log_decay", "state_in", "state_out", "offsets", "stream_ids", "workspace")] +
                [("workspace_bytes", C.c_size_t)])


class _Rows(C.Structure):
    _fields_ = [("base", C.c_void_p), ("row_stride", C.c_int64)]


class _Quantize(C.Structure):
    _fields_ = [("precision", C.c_int), ("cols", C.c_int), ("n_rows", C.c_int64), ("x", _Rows), ("codes", C.c_void_p), ("scales", C.c_void_p)]


class _Project(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("precision", "out_precision", "cols", "n_out")] + [("n_rows", C.c_int64), ("x", _Rows), ("out", _Rows)] +
                [(n, C.c_void_p) for n in ("x_scales", "weights", "weight_scales", "bias", "workspace")] + [("workspace_bytes", C.c_size_t)])


class _NibbleRing(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_codes", "k_scales", "v_codes", "v_scales")]


class _NibbleAppend(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("precision", "heads_kv", "head_dim", "rotary_dim", "interleaved")] +
                [("n_tokens", C.c_int64), ("max_tokens", C.c_int64), ("n_segments", C.c_int), ("n_streams", C.c_int), ("slots", C.c_int64),
                 ("sinks", C.c_int), ("amplitude", C.c_double), ("eps", C.c_double), ("k", _Tokens), ("v", _Tokens), ("ring", _NibbleRing)] +
                [(n, C.c_void_p) for n in ("frequencies", "k_weight", "offsets", "starts", "stream_ids")])


class _NibbleAttend(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("precision", "heads_q", "heads_kv", "head_dim")] +
                [("n_tokens", C.c_int64), ("max_tokens", C.c_int64), ("n_segments", C.c_int), ("n_streams", C.c_int), ("slots", C.c_int64),
                 ("window", C.c_int), ("sinks", C.c_int), ("scale", C.c_float), ("q", _Tokens), ("out", _Tokens), ("ring", _NibbleRing)] +
                [(n, C.c_void_p) for n in ("offsets", "starts", "stream_ids", "workspace")] + [("workspace_bytes", C.c_size_t)])


class _NibbleValues(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("precision", "heads_kv", "head_dim", "n_streams")] +
                [("slots", C.c_int64), ("ring", _NibbleRing), ("k", C.c_void_p), ("v", C.c_void_p)])


_GATE_SIZES = [("precision", C.c_int), ("channels", C.c_int), ("n_tokens", C.c_int64), ("max_tokens", C.c_int64), ("n_segments", C.c_int), ("n_streams", C.c_int)]


class _GateScan(C.Structure):
    _fields_ = (_GATE_SIZES + [(n, _Rows) for n in ("x", "gates", "out")] +
                [(n, C.c_void_p) for n in ("state_in", "state_out", "marks", "offsets", "stream_ids", "workspace")] + [("workspace_bytes", C.c_size_t), ("clear_rows", C.c_int)])


class _GateScanBackward(C.Structure):
    _fields_ = (_GATE_SIZES + [(n, _Rows) for n in ("x", "gates", "grad_out", "grad_x", "grad_gates")] +
                [(n, C.c_void_p) for n in ("grad_end", "grad_state", "marks", "offsets", "stream_ids", "workspace")] + [("workspace_bytes", C.c_size_t)])


def _direct(name, q, *args):
    """The call by way of compiled code: its outputs, or None where the arguments are not plain tensors and numbers of the usual kinds, or
    are wrong: those go the long way round, by ctypes, which converts them or raises."""
    global _native, _current_stream
    if _native is None:
        import torch
        _native, _current_stream = load_tokens(), torch._C._cuda_getCurrentRawStream
    if not getattr(q, "is_cuda", False):
        return None
    r = getattr(_native, name)(_current_stream(q.get_device()), q, *args)
    if type(r) is int:
        _check(r)
    return r


def _no_gradients(**tensors):
    import torch
    for what, t in tensors.items():
        if torch.is_grad_enabled() and getattr(t, "requires_grad", False):
            raise ValueError(f"{what} requires gradients, and there is no backward pass: detach it, or call under torch.no_grad()")
        if isinstance(t, torch.Tensor) and torch.autograd.forward_ad.unpack_dual(t).tangent is not None:
            raise ValueError(f"{what} carries a tangent, and results have none: unpack it first")


def _precision(t):
    if not _PREC:
        import torch
        _PREC.update({torch.float32: 0, torch.bfloat16: 1})
    return _PREC.get(t.dtype, -1)


def _tokens(t):
    return _Tokens(t.data_ptr(), t.stride(0), t.stride(1))


def _plain(t, dtype, shape, device, what):
    """A contiguous tensor of this type, shape and device; None stays None."""
    if t is None:
        return None
    if t.dtype != dtype or t.device != device or (shape is not None and tuple(t.shape) != tuple(shape)):
        raise ValueError(f"{what}: {t.dtype} {tuple(t.shape)} on {t.device}, wanted {dtype} {'' if shape is None else tuple(shape)} on {device}")
    return t.contiguous()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _rows(t, like, what, aligned=True):
    """Packed tokens as the library reads them: of like's type and device; copied where their rows are not to its liking."""
    if t.dim() != 3 or t.dtype != like.dtype or t.device != like.device or not t.is_cuda:
        raise ValueError(f"{what}: {t.dtype} {tuple(t.shape)} on {t.device}")
    vl = 16 // t.element_size()
    if t.stride(2) != 1 and t.shape[2] > 1 or aligned and (t.data_ptr() % 16 or t.stride(0) % vl or t.stride(1) % vl):
        t = t.contiguous()
        if aligned and t.data_ptr() % 16:
            t = t.clone()
    return t


def _out(out, shape, like, what, aligned=True):
    import torch
    if out is None:
        return torch.empty(shape, dtype=like.dtype, device=like.device)
    vl = 16 // out.element_size()
    if tuple(out.shape) != tuple(shape) or out.dtype != like.dtype or out.device != like.device or (shape[2] > 1 and out.stride(2) != 1) or \
            aligned and (out.data_ptr() % 16 or out.stride(0) % vl or out.stride(1) % vl):
        raise ValueError(f"{what}: {out.dtype} {tuple(out.shape)} with strides {out.stride()} on {out.device}")
    return out


def _written(*tensors):
    """What a call has written into tensors of the caller's counts as a change in place: torch refuses gradients that would start from what they held before."""
    import torch
    torch.autograd.graph.increment_version([t for t in tensors if t is not None])


def _stream(t):
    import torch
    return C.c_void_p(torch.cuda.current_stream(t.device).cuda_stream)


def rotary_frequencies(rotary_dim, base=10000.0, scaling=None, factor=1.0, trained=4096, fast=32.0, slow=1.0, device=None):
    """(frequencies, amplitude) of a rotation, plain or stretched for longer contexts (idf_rotary_frequencies); scaling None, "linear",
    "base" or "parts".  frequencies: float64 tensor on `device`."""
    import torch
    if scaling not in SCALING:
        raise ValueError(f"scaling {scaling!r}")
    f = np.zeros(max(1, rotary_dim // 2), dtype=np.float64)
    amplitude = C.c_double()
    _check(load_library().idf_rotary_frequencies(rotary_dim, C.c_double(base), SCALING[scaling], C.c_double(factor), C.c_double(trained),
                                                 C.c_double(fast), C.c_double(slow), C.c_void_p(f.ctypes.data), C.byref(amplitude)))
    return torch.from_numpy(f).to(device if device is not None else "cpu"), amplitude.value


def norm_rotate(q, k, positions, frequencies, layout="half", amplitude=1.0, q_weight=None, k_weight=None, eps=1e-6, q_out=None, k_out=None):
    """Queries [token][head][value] and keys of the same tokens, each head normalised (where there is a weight) and turned by its token's
    position: (q, k) anew, or into q_out and k_out, which may be q and k (idf_norm_rotate).  layout "half" or "interleaved"."""
    if layout not in ("half", "interleaved"):
        raise ValueError(f"layout {layout!r}")
    r = _direct("norm_rotate", q, k, positions, frequencies, int(layout == "interleaved"), amplitude, q_weight, k_weight, eps, q_out, k_out)
    return r if r is not None else _norm_rotate(q, k, positions, frequencies, layout, amplitude, q_weight, k_weight, eps, q_out, k_out)


def _norm_rotate(q, k, positions, frequencies, layout, amplitude, q_weight, k_weight, eps, q_out, k_out):
    import torch
    _no_gradients(q=q, k=k, frequencies=frequencies, q_weight=q_weight, k_weight=k_weight, q_out=q_out, k_out=k_out)
    q, k = _rows(q, q, "q", aligned=False), _rows(k, q, "k", aligned=False)
    n, hq, d = q.shape
    if k.shape[0] != n or k.shape[2] != d:
        raise ValueError(f"queries {tuple(q.shape)} and keys {tuple(k.shape)}")
    q_out, k_out = _out(q_out, q.shape, q, "q_out", aligned=False), _out(k_out, k.shape, q, "k_out", aligned=False)
    positions = _plain(positions, torch.int64, (n,), q.device, "positions")
    frequencies = _plain(frequencies, torch.float64, None, q.device, "frequencies")
    q_weight, k_weight = (_plain(w, torch.float32, (d,), q.device, "weight") for w in (q_weight, k_weight))
    a = _NormRotate(_precision(q), hq, k.shape[1], d, 2 * frequencies.numel(), int(layout == "interleaved"), n, _tokens(q), _tokens(k),
                    _tokens(q_out), _tokens(k_out), _ptr(positions), _ptr(frequencies), _ptr(q_weight), _ptr(k_weight), amplitude, eps)
    with torch.cuda.device(q.device):
        _check(load_library().idf_norm_rotate(C.byref(a), _stream(q)))
    _written(q_out, k_out)
    return q_out, k_out


def _segments(n, offsets, max_tokens, n_segments, device):
    """(offsets, longest segment, segments)"""
    import torch
    if offsets is None:
        if n_segments == 0 or n % n_segments:
            if n:
                raise ValueError(f"{n} tokens are not {n_segments} segments of one length")
            return None, 0, n_segments
        return None, n // n_segments, n_segments
    if max_tokens is None:
        raise ValueError("offsets without max_tokens: the longest segment is not known to the host")
    offsets = _plain(offsets, torch.int64, None, device, "offsets")
    return offsets, max_tokens, offsets.numel() - 1


def _workspace(fn, a, device):
    import torch
    nb = C.c_size_t()
    _check(fn(C.byref(a), C.byref(nb)))
    if nb.value == 0:
        return None
    ws = torch.empty(nb.value, dtype=torch.uint8, device=device)
    a.workspace, a.workspace_bytes = ws.data_ptr(), nb.value
    return ws


def window_attend(q, k, v, k_ring=None, v_ring=None, starts=None, *, window, sinks=0, scale=None, offsets=None, max_tokens=None,
                  stream_ids=None, out=None):
    """Attention of packed segments over the last `window` tokens of their streams and the first `sinks` ones, which the rings
    [stream][slot][head][value] hold; the segments' keys and values are written to the rings (idf_window_attend).

    starts: int64, position of each segment's first token.  Without offsets all segments have one length; with offsets (int64, one more
    than segments) max_tokens is the longest one's.  stream_ids: int32, the ring of each segment.  scale: 1 / sqrt(head size)."""
    r = _direct("window_attend", q, k, v, k_ring, v_ring, starts, window, sinks, scale, offsets, max_tokens, stream_ids, out)
    return r if r is not None else _window_attend(q, k, v, k_ring, v_ring, starts, window, sinks, scale, offsets, max_tokens, stream_ids, out)


def _window_attend(q, k, v, k_ring, v_ring, starts, window, sinks, scale, offsets, max_tokens, stream_ids, out):
    import torch
    _no_gradients(q=q, k=k, v=v, k_ring=k_ring, v_ring=v_ring, out=out)
    q, k, v = _rows(q, q, "q"), _rows(k, q, "k"), _rows(v, q, "v")
    n, hq, d = q.shape
    hkv = k.shape[1]
    if k.shape != v.shape or k.shape[0] != n or k.shape[2] != d:
        raise ValueError(f"queries {tuple(q.shape)}, keys {tuple(k.shape)} and values {tuple(v.shape)}")
    streams = slots = 0
    if k_ring is not None or v_ring is not None:
        if k_ring is None or v_ring is None:
            raise ValueError("a ring of keys or values alone")
        for r in (k_ring, v_ring):
            if r.dim() != 4 or r.dtype != q.dtype or r.device != q.device or not r.is_contiguous() or r.shape != k_ring.shape or tuple(r.shape[2:]) != (hkv, d):
                raise ValueError(f"ring: {r.dtype} {tuple(r.shape)} on {r.device}, wanted contiguous {q.dtype} [streams][slots][{hkv}][{d}]")
        streams, slots = k_ring.shape[:2]
    n_segments = next((t.numel() for t in (stream_ids, starts) if t is not None), streams if k_ring is not None else 1)
    offsets, longest, n_segments_ = _segments(n, offsets, max_tokens, n_segments, q.device)
    if offsets is not None and n_segments_ != n_segments and (stream_ids is not None or starts is not None):
        raise ValueError(f"{n_segments_} segments by offsets, {n_segments} by starts or stream_ids")
    n_segments = n_segments_
    starts = _plain(starts, torch.int64, (n_segments,), q.device, "starts")
    stream_ids = _plain(stream_ids, torch.int32, (n_segments,), q.device, "stream_ids")
    out = _out(out, q.shape, q, "out")
    a = _Window(_precision(q), hq, hkv, d, n, longest, n_segments, streams if k_ring is not None else n_segments, slots, window, sinks,
                1.0 / math.sqrt(d) if scale is None else scale, _tokens(q), _tokens(k), _tokens(v), _tokens(out), _ptr(k_ring), _ptr(v_ring),
                _ptr(offsets), _ptr(starts), _ptr(stream_ids), None, 0)
    L = load_library()
    with torch.cuda.device(q.device):
        ws = _workspace(L.idf_window_workspace, a, q.device)          # noqa: F841 (held until the work is enqueued)
        _check(L.idf_window_attend(C.byref(a), _stream(q)))
    _written(out, k_ring, v_ring)
    return out


def decay_attend(q, k, v, log_decay, state=None, state_out=None, *, scale=None, offsets=None, max_tokens=None, n_segments=None,
                 stream_ids=None, out=None):
    """Linear attention of packed segments with a decay per key/value head, from `state` (float32 [stream][head][key value][value], None:
    zeros) into `state_out` (None: not wanted; may be `state`) (idf_decay_attend).  Segments as in window_attend; n_segments where
    neither states nor ids say how many there are.  scale: 1 / sqrt(key size)."""
    r = _direct("decay_attend", q, k, v, log_decay, state, state_out, scale, offsets, max_tokens, n_segments, stream_ids, out)
    return r if r is not None else _decay_attend(q, k, v, log_decay, state, state_out, scale, offsets, max_tokens, n_segments, stream_ids, out)


def _decay_attend(q, k, v, log_decay, state, state_out, scale, offsets, max_tokens, n_segments, stream_ids, out):
    import torch
    _no_gradients(q=q, k=k, v=v, log_decay=log_decay, state=state, state_out=state_out, out=out)
    q, k, v = _rows(q, q, "q"), _rows(k, q, "k"), _rows(v, q, "v")
    n, hq, dk = q.shape
    hkv, dv = v.shape[1:]
    if tuple(k.shape) != (n, hkv, dk) or v.shape[0] != n:
        raise ValueError(f"queries {tuple(q.shape)}, keys {tuple(k.shape)} and values {tuple(v.shape)}")
    streams = None
    for s in (state, state_out):
        if s is None:
            continue
        if s.dim() != 4 or s.dtype != torch.float32 or s.device != q.device or not s.is_contiguous() or tuple(s.shape[1:]) != (hkv, dk, dv) or streams not in (None, s.shape[0]):
            raise ValueError(f"state: {s.dtype} {tuple(s.shape)} on {s.device}, wanted contiguous float32 [streams][{hkv}][{dk}][{dv}]")
        streams = s.shape[0]
    count = next((c for c in (None if stream_ids is None else stream_ids.numel(), n_segments, streams) if c is not None), 1)
    offsets, longest, n_segments_ = _segments(n, offsets, max_tokens, count, q.device)
    if offsets is not None and n_segments_ != count and (stream_ids is not None or n_segments is not None):
        raise ValueError(f"{n_segments_} segments by offsets, {count} by stream_ids or n_segments")
    stream_ids = _plain(stream_ids, torch.int32, (n_segments_,), q.device, "stream_ids")
    log_decay = _plain(log_decay, torch.float32, (hkv,), q.device, "log_decay")
    out = _out(out, (n, hq, dv), q, "out")
    a = _Decay(_precision(q), hq, hkv, dk, dv, n, longest, n_segments_, n_segments_ if streams is None else streams,
               1.0 / math.sqrt(dk) if scale is None else scale, _tokens(q), _tokens(k), _tokens(v), _tokens(out), _ptr(log_decay),
               _ptr(state), _ptr(state_out), _ptr(offsets), _ptr(stream_ids), None, 0)
    L = load_library()
    with torch.cuda.device(q.device):
        ws = _workspace(L.idf_decay_workspace, a, q.device)           # noqa: F841 (held until the work is enqueued)
        _check(L.idf_decay_attend(C.byref(a), _stream(q)))
    _written(out, state_out)
    return out


# ---- in few bits, and a recurrence per channel ----

def _matrix(t, like, what, dtype=None):
    """Rows as the library reads them, of like's device; copied where their values lie apart, or rows further than it takes."""
    if t.dim() != 2 or t.dtype != (like.dtype if dtype is None else dtype) or t.device != like.device or not t.is_cuda:
        raise ValueError(f"{what}: {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.contiguous() if t.shape[1] > 1 and t.stride(1) != 1 or t.shape[0] > 1 and t.stride(0) > 1 << 25 else t


def _as_rows(t):
    return _Rows(t.data_ptr(), t.stride(0) if t.shape[0] > 1 else t.shape[1])


def _out_matrix(out, shape, dtype, device, what):
    import torch
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if tuple(out.shape) != tuple(shape) or out.device != device or shape[1] > 1 and out.stride(1) != 1:
        raise ValueError(f"{what}: {out.dtype} {tuple(out.shape)} with strides {out.stride()} on {out.device}, wanted {tuple(shape)} on {device}")
    return out


def _share(a, b):
    """Whether two matrices (or rows) share places: where their rows lie alike they may be columns of one larger matrix, else it is enough that they reach into each other."""
    if not a.numel() or not b.numel():
        return False
    (rows_a, wide_a), (rows_b, wide_b) = ((t.numel() // t.shape[-1], t.shape[-1] * t.element_size()) for t in (a, b))
    strides = [t.stride(0) * t.element_size() if t.dim() == 2 else 0 for t in (a, b)]
    strides = [s if rows > 1 else 0 for s, rows in zip(strides, (rows_a, rows_b))]
    apart = b.data_ptr() - a.data_ptr()
    if not -(rows_b - 1) * strides[1] - wide_b < apart < (rows_a - 1) * strides[0] + wide_a:
        return False
    stride = max(strides)
    if any(s != stride for s, rows in zip(strides, (rows_a, rows_b)) if rows > 1) or max(wide_a, wide_b) > stride:
        return True
    # row j of b begins `rest` behind row j + k of a
    k, rest = divmod(apart, stride)
    both = [max(0, -d) < min(rows_b, rows_a - d) for d in (k, k + 1)]
    return (both[0] and rest < wide_a) or (both[1] and stride - rest < wide_b)


def quantize_rows(x, codes=None, scales=None):
    """Rows of a matrix in 8 bits with a scale each: (codes, int8 [rows][columns rounded up to 16, zeros behind them], scales float32 [rows])
    (idf_quantize_rows).  For tokens, and for the rows of a matrix of weights [outputs][columns]."""
    r = _direct("quantize_rows", x, codes, scales)
    return r if r is not None else _quantize_rows(x, codes, scales)


def _quantize_rows(x, codes, scales):
    import torch
    _no_gradients(x=x)
    x = _matrix(x, x, "x")
    rows, cols = x.shape
    padded = -(-cols // 16) * 16
    for t, dtype, shape in ((codes, torch.int8, (rows, padded)), (scales, torch.float32, (rows,))):
        if t is not None and (t.dtype != dtype or tuple(t.shape) != shape or t.device != x.device or not t.is_contiguous()):
            raise ValueError(f"{t.dtype} {tuple(t.shape)} on {t.device}, wanted contiguous {dtype} {shape} on {x.device}")
    codes = torch.empty(rows, padded, dtype=torch.int8, device=x.device) if codes is None else codes
    scales = torch.empty(rows, dtype=torch.float32, device=x.device) if scales is None else scales
    a = _Quantize(_precision(x), cols, rows, _as_rows(x), _ptr(codes), _ptr(scales))
    with torch.cuda.device(x.device):
        _check(load_library().idf_quantize_rows(C.byref(a), _stream(x)))
    _written(codes, scales)
    return codes, scales


def project_rows(x, weight, weight_scales, bias=None, x_scales=None, dtype=None, out=None):
    """x [rows][columns] times the transpose of a matrix of 8-bit weights [outputs][columns rounded up to 16] with a scale for each output, plus a bias
    (idf_project_rows).  x in float32 or bfloat16 is taken to 8 bits with a scale for each row on the way; in int8 it comes with its
    x_scales, and dtype or out says what the result is in (else what x is in).  out may lie beside what is read, not over it."""
    import torch
    to_f32 = {None: -1, torch.float32: 1, torch.bfloat16: 0}.get(dtype)
    r = None if to_f32 is None else _direct("project_rows", x, weight, weight_scales, bias, x_scales, to_f32, out)
    return r if r is not None else _project_rows(x, weight, weight_scales, bias, x_scales, dtype, out)


def _project_rows(x, weight, weight_scales, bias, x_scales, dtype, out):
    import torch
    _no_gradients(x=x, weight_scales=weight_scales, bias=bias, x_scales=x_scales, out=out)
    x = _matrix(x, x, "x")
    coded = x.dtype == torch.int8
    if coded != (x_scales is not None):
        raise ValueError("x_scales go with x in int8")
    if coded and dtype is None and out is None:
        raise ValueError("x in int8 does not say what the result is in: dtype or out")
    if coded and (x.data_ptr() % 16 or x.shape[0] > 1 and x.stride(0) % 16):
        x = x.contiguous()
        x = x.clone() if x.data_ptr() % 16 else x
    rows, cols = x.shape
    padded = -(-cols // 16) * 16
    if weight.dim() != 2 or weight.shape[1] != padded:
        raise ValueError(f"weight {tuple(weight.shape)}, wanted [outputs][{padded}] for rows of {cols}")
    weight = _plain(weight, torch.int8, None, x.device, "weight")
    weight = weight.clone() if weight.data_ptr() % 16 else weight
    n = weight.shape[0]
    weight_scales, bias = (_plain(t, torch.float32, (n,), x.device, what) for t, what in ((weight_scales, "weight_scales"), (bias, "bias")))
    x_scales = _plain(x_scales, torch.float32, (rows,), x.device, "x_scales")
    out = _out_matrix(out, (rows, n), x.dtype if dtype is None else dtype, x.device, "out")
    if dtype is not None and out.dtype != dtype:
        raise ValueError(f"out: {out.dtype}, wanted {dtype}")
    if any(t is not None and _share(out, t) for t in (x, weight, weight_scales, bias, x_scales)):
        raise ValueError("out shares places with what is read")
    a = _Project(2 if coded else _precision(x), _precision(out), cols, n, rows, _as_rows(x), _as_rows(out), _ptr(x_scales), _ptr(weight),
                 _ptr(weight_scales), _ptr(bias), None, 0)
    L = load_library()
    with torch.cuda.device(x.device):
        ws = _workspace(L.idf_project_workspace, a, x.device)         # noqa: F841 (held until the work is enqueued)
        _check(L.idf_project_rows(C.byref(a), _stream(x)))
    _written(out)
    return out


class NibbleRing(NamedTuple):
    """A ring of keys and values in 4 bits (idf_nibble_ring): codes, uint8 [stream][head][slot][head size / 2], and powers of two,
    uint8 [stream][head][slot][head size / 32]."""
    k_codes: object
    k_scales: object
    v_codes: object
    v_scales: object


def nibble_ring(n_streams, slots, heads, dim, device="cuda:0"):
    """An empty NibbleRing: 17 bytes for 32 values."""
    import torch
    if dim % 32 or not 32 <= dim <= 256:
        raise ValueError(f"heads of {dim} values: multiples of 32 up to 256")
    return NibbleRing(*(torch.zeros(n_streams, heads, slots, dim // by, dtype=torch.uint8, device=device) for by in (2, 32, 2, 32)))


def _nibble_ring(ring, device=None):
    """(the library's ring, streams, heads, slots, head size)"""
    import torch
    codes = ring[0]
    for i, t in enumerate(ring):
        if t.dtype != torch.uint8 or t.dim() != 4 or not t.is_contiguous() or not t.is_cuda or t.device != (codes.device if device is None else device) or \
                t.shape[:3] != codes.shape[:3] or t.shape[3] * (16 if i % 2 else 1) != codes.shape[3]:
            raise ValueError(f"ring: {t.dtype} {tuple(t.shape)} on {t.device}, wanted contiguous uint8 [streams][heads][slots][dim / 2] and [..][dim / 32]")
    _no_gradients(**dict(zip(NibbleRing._fields, ring)))
    streams, heads, slots, half = codes.shape
    return _NibbleRing(*(t.data_ptr() for t in ring)), streams, heads, slots, 2 * half


def _places(n, streams, starts, offsets, max_tokens, stream_ids, device):
    """(offsets, longest segment, segments, starts, stream_ids)"""
    import torch
    count = next((t.numel() for t in (stream_ids, starts) if t is not None), streams)
    offsets, longest, n_segments = _segments(n, offsets, max_tokens, count, device)
    if offsets is not None and n_segments != count and (stream_ids is not None or starts is not None):
        raise ValueError(f"{n_segments} segments by offsets, {count} by starts or stream_ids")
    return (offsets, longest, n_segments, _plain(starts, torch.int64, (n_segments,), device, "starts"),
            _plain(stream_ids, torch.int32, (n_segments,), device, "stream_ids"))


def nibble_append(k, v, ring, starts=None, *, sinks=0, frequencies=None, layout="half", amplitude=1.0, k_weight=None, eps=1e-6, offsets=None,
                 max_tokens=None, stream_ids=None):
    """Segments' keys and values [token][head][value] into their streams' rings of 4-bit blocks, keys normalised (where there is a weight) and turned by
    position (where there are frequencies) on the way, as norm_rotate does it to queries (idf_nibble_append).  Segments as in window_attend."""
    if layout not in ("half", "interleaved"):
        raise ValueError(f"layout {layout!r}")
    r = _direct("nibble_append", k, v, *ring, starts, sinks, frequencies, int(layout == "interleaved"), amplitude, k_weight, eps, offsets, max_tokens, stream_ids)
    if r is None:
        _nibble_append(k, v, ring, starts, sinks, frequencies, layout, amplitude, k_weight, eps, offsets, max_tokens, stream_ids)


def _nibble_append(k, v, ring, starts, sinks, frequencies, layout, amplitude, k_weight, eps, offsets, max_tokens, stream_ids):
    import torch
    _no_gradients(k=k, v=v, frequencies=frequencies, k_weight=k_weight)
    k, v = _rows(k, k, "k", aligned=False), _rows(v, k, "v", aligned=False)
    held, streams, heads, slots, dim = _nibble_ring(ring, k.device)
    n = k.shape[0]
    if k.shape != v.shape or tuple(k.shape[1:]) != (heads, dim):
        raise ValueError(f"keys {tuple(k.shape)} and values {tuple(v.shape)} for a ring of {heads} heads of {dim}")
    offsets, longest, n_segments, starts, stream_ids = _places(n, streams, starts, offsets, max_tokens, stream_ids, k.device)
    frequencies = _plain(frequencies, torch.float64, None, k.device, "frequencies")
    k_weight = _plain(k_weight, torch.float32, (dim,), k.device, "k_weight")
    a = _NibbleAppend(_precision(k), heads, dim, 0 if frequencies is None else 2 * frequencies.numel(), int(layout == "interleaved"), n, longest, n_segments,
                     streams, slots, sinks, amplitude, eps, _tokens(k), _tokens(v), held, _ptr(frequencies), _ptr(k_weight), _ptr(offsets), _ptr(starts),
                     _ptr(stream_ids))
    with torch.cuda.device(k.device):
        _check(load_library().idf_nibble_append(C.byref(a), _stream(k)))
    _written(*ring)


def nibble_attend(q, ring, starts=None, *, window, sinks=0, scale=None, offsets=None, max_tokens=None, stream_ids=None, out=None):
    """Attention of packed segments' queries over the last `window` tokens of their streams and the first `sinks` ones, their own among them, which have been
    appended to the rings of 4-bit blocks before (idf_nibble_attend); a ring has room for a segment beside a window.  starts: int64, position of each
    segment's first query; segments as in window_attend.  scale: 1 / sqrt(head size)."""
    r = _direct("nibble_attend", q, *ring, starts, window, sinks, scale, offsets, max_tokens, stream_ids, out)
    return r if r is not None else _nibble_attend(q, ring, starts, window, sinks, scale, offsets, max_tokens, stream_ids, out)


def _nibble_attend(q, ring, starts, window, sinks, scale, offsets, max_tokens, stream_ids, out):
    import torch
    _no_gradients(q=q, out=out)
    q = _rows(q, q, "q")
    held, streams, heads, slots, dim = _nibble_ring(ring, q.device)
    n, hq = q.shape[:2]
    if q.shape[2] != dim:
        raise ValueError(f"queries {tuple(q.shape)} for a ring of {heads} heads of {dim}")
    offsets, longest, n_segments, starts, stream_ids = _places(n, streams, starts, offsets, max_tokens, stream_ids, q.device)
    out = _out(out, q.shape, q, "out")
    a = _NibbleAttend(_precision(q), hq, heads, dim, n, longest, n_segments, streams, slots, window, sinks, 1.0 / math.sqrt(dim) if scale is None else scale,
                     _tokens(q), _tokens(out), held, _ptr(offsets), _ptr(starts), _ptr(stream_ids), None, 0)
    L = load_library()
    with torch.cuda.device(q.device):
        ws = _workspace(L.idf_nibble_attend_workspace, a, q.device)    # noqa: F841 (held until the work is enqueued)
        _check(L.idf_nibble_attend(C.byref(a), _stream(q)))
    _written(out)
    return out


def nibble_values(ring, dtype=None):
    """(keys, values) that a NibbleRing stands for, [stream][slot][head][value] in bfloat16 (or float32): rings as window_attend takes them
    (idf_nibble_values)."""
    import torch
    if dtype not in (None, torch.float32, torch.bfloat16):
        raise ValueError(f"values in {dtype}: float32 or bfloat16")
    r = _direct("nibble_values", *ring, int(dtype == torch.float32))
    return r if r is not None else _nibble_values(ring, torch.bfloat16 if dtype is None else dtype)


def _nibble_values(ring, dtype):
    import torch
    held, streams, heads, slots, dim = _nibble_ring(ring)
    k, v = (torch.empty(streams, slots, heads, dim, dtype=dtype, device=ring[0].device) for _ in range(2))
    a = _NibbleValues(_precision(k), heads, dim, streams, slots, held, _ptr(k), _ptr(v))
    with torch.cuda.device(k.device):
        _check(load_library().idf_nibble_values(C.byref(a), _stream(k)))
    return k, v


def _gate_sizes(x, gates, states, offsets, max_tokens, n_segments, stream_ids, n_streams=None):
    """What the structures of the recurrence begin with, and offsets and stream_ids."""
    import torch
    n, channels = x.shape
    if gates.shape != x.shape:
        raise ValueError(f"x {tuple(x.shape)} and gates {tuple(gates.shape)}")
    for s in states:
        if s is None:
            continue
        if s.dim() != 2 or s.dtype != torch.float32 or s.device != x.device or not s.is_contiguous() or s.shape[1] != channels or n_streams not in (None, s.shape[0]):
            raise ValueError(f"state: {s.dtype} {tuple(s.shape)} on {s.device}, wanted contiguous float32 [streams][{channels}]")
        n_streams = s.shape[0]
    count = next((c for c in (None if stream_ids is None else stream_ids.numel(), n_segments, n_streams) if c is not None), 1)
    offsets, longest, n_segments_ = _segments(n, offsets, max_tokens, count, x.device)
    if offsets is not None and n_segments_ != count and (stream_ids is not None or n_segments is not None):
        raise ValueError(f"{n_segments_} segments by offsets, {count} by stream_ids or n_segments")
    stream_ids = _plain(stream_ids, torch.int32, (n_segments_,), x.device, "stream_ids")
    return (_precision(x), channels, n, longest, n_segments_, n_segments_ if n_streams is None else n_streams), offsets, stream_ids


def _marks_floats(sizes, offsets):
    a, nb = _GateScan(*sizes), C.c_size_t()
    a.offsets = _ptr(offsets)
    _check(load_library().idf_gate_scan_marks(C.byref(a), C.byref(nb)))
    return nb.value // 4


def gate_scan(x, gates, state=None, state_out=None, *, offsets=None, max_tokens=None, n_segments=None, stream_ids=None, out=None, marks=None):
    """h = a h + (1 - a) x per channel along the tokens of packed segments, a = sigmoid(gates): x, gates and the result [token][channel], from `state` (float32
    [stream][channel], None: zeros) into `state_out` (None: not wanted; may be `state`) (idf_gate_scan).  Segments as in decay_attend; rows that none of them
    has are zeros in a new result, and stay as they are in `out`.
    marks True: returns (out, marks), the latter for gate_scan_backward.  gate_scan_recorded is the form that torch's gradients go through."""
    r = _direct("gate_scan", x, gates, state, state_out, offsets, max_tokens, n_segments, stream_ids, out, marks)
    return r if r is not None else _gate_scan(x, gates, state, state_out, offsets, max_tokens, n_segments, stream_ids, out, marks)


def _gate_scan(x, gates, state, state_out, offsets, max_tokens, n_segments, stream_ids, out, marks):
    import torch
    _no_gradients(x=x, gates=gates, state=state, state_out=state_out, out=out)
    x, gates = _matrix(x, x, "x"), _matrix(gates, x, "gates")
    sizes, offsets, stream_ids = _gate_sizes(x, gates, (state, state_out), offsets, max_tokens, n_segments, stream_ids)
    clear = out is None and offsets is not None    # (a new result holds nothing yet)
    out = _out_matrix(out, x.shape, x.dtype, x.device, "out")
    if out.dtype != x.dtype:
        raise ValueError(f"out: {out.dtype}, wanted {x.dtype}")
    if _share(out, x) or _share(out, gates):
        raise ValueError("out shares places with x or gates")
    given = marks
    if marks is not None:
        marks = torch.empty(_marks_floats(sizes, offsets), device=x.device) if marks is True else _plain(marks, torch.float32, (_marks_floats(sizes, offsets),), x.device, "marks")
        if given is not True and marks is not given:
            raise ValueError("marks have to be contiguous")
    a = _GateScan(*sizes, _as_rows(x), _as_rows(gates), _as_rows(out), _ptr(state), _ptr(state_out), _ptr(marks), _ptr(offsets), _ptr(stream_ids), None, 0, clear)
    L = load_library()
    with torch.cuda.device(x.device):
        ws = _workspace(L.idf_gate_scan_workspace, a, x.device)       # noqa: F841 (held until the work is enqueued)
        _check(L.idf_gate_scan(C.byref(a), _stream(x)))
    _written(out, state_out, marks)
    return (out, marks) if given is True else out


def gate_scan_backward(x, gates, marks, grad_out=None, grad_end=None, *, offsets=None, max_tokens=None, n_segments=None, stream_ids=None, n_streams=None):
    """Gradients of gate_scan's x, gates and state from those of its result and of state_out (None: zeros), with the marks that the call left
    (idf_gate_scan_backward).  n_streams where grad_end does not say how many there are; streams that no segment is of get zeros."""
    r = _direct("gate_scan_backward", x, gates, marks, grad_out, grad_end, offsets, max_tokens, n_segments, stream_ids, n_streams)
    return r if r is not None else _gate_scan_backward(x, gates, marks, grad_out, grad_end, offsets, max_tokens, n_segments, stream_ids, n_streams)


def _gate_scan_backward(x, gates, marks, grad_out, grad_end, offsets, max_tokens, n_segments, stream_ids, n_streams):
    import torch
    _no_gradients(x=x, gates=gates, grad_out=grad_out, grad_end=grad_end)
    x, gates = _matrix(x, x, "x"), _matrix(gates, x, "gates")
    sizes, offsets, stream_ids = _gate_sizes(x, gates, (grad_end,), offsets, max_tokens, n_segments, stream_ids, n_streams)
    if grad_out is not None:
        grad_out = _matrix(grad_out, x, "grad_out")
        if grad_out.shape != x.shape:
            raise ValueError(f"grad_out {tuple(grad_out.shape)} of x {tuple(x.shape)}")
    marks = _plain(marks, torch.float32, (_marks_floats(sizes, offsets),), x.device, "marks")
    grads = [torch.empty(x.shape, dtype=x.dtype, device=x.device) for _ in range(2)]
    grad_state = torch.zeros(sizes[5], x.shape[1], device=x.device)        # (streams that no segment is of have no gradient here)
    a = _GateScanBackward(*sizes, _as_rows(x), _as_rows(gates), _Rows(None, 0) if grad_out is None else _as_rows(grad_out), *(_as_rows(t) for t in grads),
                          _ptr(grad_end), _ptr(grad_state), _ptr(marks), _ptr(offsets), _ptr(stream_ids), None, 0)
    L = load_library()
    with torch.cuda.device(x.device):
        ws = _workspace(L.idf_gate_scan_backward_workspace, a, x.device)          # noqa: F841 (held until the work is enqueued)
        _check(L.idf_gate_scan_backward(C.byref(a), _stream(x)))
    return *grads, grad_state


_recorded = None             # the autograd function, made with the first call


def _make_recorded():
    import torch
    from torch.autograd.function import once_differentiable

    class GateScan(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, gates, state, offsets, max_tokens, n_segments):
            streams = n_segments if n_segments is not None else offsets.numel() - 1 if offsets is not None else 1 if state is None else state.shape[0]
            if state is not None and state.shape[0] != streams:
                raise ValueError(f"{state.shape[0]} states of {streams} segments")
            end = torch.empty(streams, x.shape[1], device=x.device)
            out, marks = gate_scan(x, gates, state, end, offsets=offsets, max_tokens=max_tokens, n_segments=n_segments, marks=True)
            ctx.save_for_backward(x, gates, marks, offsets)
            ctx.sizes = max_tokens, n_segments, streams
            ctx.set_materialize_grads(False)
            return out, end

        @staticmethod
        @once_differentiable
        def backward(ctx, grad_out, grad_end):
            if grad_out is None and grad_end is None:
                return (None,) * 6
            x, gates, marks, offsets = ctx.saved_tensors
            max_tokens, n_segments, streams = ctx.sizes
            _no_capture(x)
            dx, dg, ds = gate_scan_backward(x, gates, marks, grad_out, None if grad_end is None else grad_end.contiguous(), offsets=offsets,
                                            max_tokens=max_tokens, n_segments=n_segments, n_streams=streams)
            need = ctx.needs_input_grad
            return dx if need[0] else None, dg if need[1] else None, ds if need[2] else None, None, None, None
    return GateScan


def _no_capture(x):
    import torch
    if not x.is_cuda:
        return
    with torch.cuda.device(x.device):              # (the stream that is asked about is the current device's)
        capturing = torch.cuda.is_current_stream_capturing()
    if capturing:
        raise RuntimeError("gate_scan_recorded while a stream is captured: torch ends the process there where leaves have recorded outside; "
                           "gate_scan with marks and gate_scan_backward can be captured")


def gate_scan_recorded(x, gates, state=None, *, offsets=None, max_tokens=None, n_segments=None):
    """gate_scan for training: (out, states behind the segments), both recorded by torch's gradients where x, gates or state require them, once (gradients
    of gradients are refused).  Segment s is of stream s; rows that no segment has are zeros.  Not for a stream that is being captured into a graph."""
    global _recorded
    r = _direct("gate_scan_recorded", x, gates, state, offsets, max_tokens, n_segments)
    if r is not None:
        return r
    _no_capture(x)
    if _recorded is None:
        _recorded = _make_recorded()
    return _recorded.apply(x, gates, state, offsets, max_tokens, n_segments)
