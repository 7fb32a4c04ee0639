"""The operators that mix the tokens of streams (include/idf.h, last section) on torch tensors: argument marshalling only.

Everything is enqueued on the current stream of the tensors' device.  There is no backward pass: tensors that require gradients are refused
where gradients are recorded, taken under torch.no_grad().  Packed tokens [token][head][value]; a tensor whose values lie
apart, or whose rows do not begin at multiples of 16 bytes where the library asks for that, is copied first.
"""
from __future__ import annotations

import ctypes as C
import math

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
    return out
