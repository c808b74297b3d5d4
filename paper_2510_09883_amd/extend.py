"""Python binding of the prompt side of libdelta_attn.so (include/delta_extend.h): rotated append of
runs of new tokens and their causal attention over the paged cache.  Argument marshalling only, in
the manner of the decode-step binding: tensors by device pointer, torch's current stream, a
non-zero status raises DeltaError.  Shapes and cache descriptors come from delta.make_shape and
delta.make_kv."""
from __future__ import annotations

import ctypes

import torch

from . import delta
from .delta import DeltaError, _check, _check_kv, _dev, _nbytes, _P, _ptr, _vp
from .delta import delta_kv_t, delta_shape_t

EXPORTED = ["delta_rope_append", "delta_extend_workspace_bytes", "delta_extend_attn"]


class delta_rope_t(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


_i32, _i64 = ctypes.c_int32, ctypes.c_int64


def _bind(lib):
    """Declare the C signatures of include/delta_extend.h on a loaded library handle."""
    lib.delta_rope_append.argtypes = [_P(delta_shape_t), _P(delta_kv_t), _P(delta_rope_t), _i32, _vp,
                                      _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp]
    lib.delta_extend_workspace_bytes.argtypes = [_P(delta_shape_t), _i32, _i32, _P(ctypes.c_size_t)]
    lib.delta_extend_attn.argtypes = [_P(delta_shape_t), _P(delta_kv_t), _i32, _i32, _vp, _vp, _vp, _vp,
                                      ctypes.c_size_t, _vp]
    for n in EXPORTED:
        getattr(lib, n).restype = ctypes.c_int
    return lib


_bind(delta._lib)   # (calls go to the library that the decode-step binding has loaded)


def _rows(name, t, heads, d):
    """A bf16 [rows, heads, d] GPU tensor whose rows may stand apart; its row stride.  What passes is
    found out first, and what does not is given its message after."""
    if type(t) is torch.Tensor and t.is_cuda and t.dtype == torch.bfloat16:
        have, stride = t.shape, t.stride()
        if have[1:] == (heads, d) and stride[1:] == (d, 1):
            return stride[0] if have[0] > 1 else heads * d   # (the stride of a single row says nothing)
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a GPU tensor (got device {t.device})")
    if t.dtype != torch.bfloat16:
        raise ValueError(f"{name}: expected {torch.bfloat16}, got {t.dtype}")
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != d:
        raise ValueError(f"{name}: expected shape {(None, heads, d)}, got {tuple(t.shape)}")
    row, head, elem = t.stride()
    if t.numel() and (elem != 1 or (head != d and heads > 1)):
        raise ValueError(f"{name}: the heads of a row must lie one behind the other")
    return heads * d if t.shape[0] < 2 else row


def _offsets(row_offsets, batch):
    if row_offsets is not None:
        _dev("row_offsets", row_offsets, torch.int32, (batch + 1,))


def _stream_of(kv, *tensors):
    """The current device's current stream; the cache and every tensor have to be on that device."""
    here = torch.cuda.current_device()
    for t in (*tensors, *getattr(kv, "_tensors", ())[:1]):
        if t is not None and t.get_device() != here:
            raise ValueError(f"tensor on {t.device}, but the current device is cuda:{here}")
    return torch._C._cuda_getCurrentRawStream(here)


def delta_rope_append(shape, kv: delta_kv_t, q, k, v, q_out, inv_freq=None, row_offsets=None,
                      positions=None, interleaved=False):
    """Rotates q and k [rows, heads, head_dim] of the new tokens (by inv_freq [rotary_dim / 2]; None:
    not at all), writes k and v to the cache and the rotated queries to q_out; q and q_out may both
    be None.  row_offsets [batch + 1]: the runs (None: one token per sequence)."""
    _check_kv(kv, shape)
    ks = _rows("k", k, shape.n_kv_heads, shape.head_dim)
    vs = _rows("v", v, shape.n_kv_heads, shape.head_dim)
    n = k.shape[0]
    if v.shape[0] != n:
        raise ValueError(f"v: {v.shape[0]} rows, but k has {n}")
    qs = 0
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out come together")
    if q is not None:
        qs = _rows("q", q, shape.n_q_heads, shape.head_dim)
        if q.shape[0] != n:
            raise ValueError(f"q: {q.shape[0]} rows, but k has {n}")
        _dev("q_out", q_out, torch.bfloat16, (n, shape.n_q_heads, shape.head_dim))
    _offsets(row_offsets, shape.batch)
    rope = None
    if inv_freq is not None:
        _dev("inv_freq", inv_freq, torch.float32, (None,))
        if positions is not None:
            _dev("positions", positions, torch.int32, (n,))
        rope = ctypes.byref(delta_rope_t(inv_freq.data_ptr(), _ptr(positions), 2 * inv_freq.shape[0],
                                         1 if interleaved else 0))
    elif positions is not None:
        raise ValueError("positions: nothing is rotated without inv_freq")
    stream = _stream_of(kv, k, v, q, q_out, row_offsets, inv_freq, positions)
    _check("delta_rope_append",
           delta._lib.delta_rope_append(ctypes.byref(shape), ctypes.byref(kv), rope, n, _ptr(row_offsets),
                                        _ptr(q), qs, k.data_ptr(), ks, v.data_ptr(), vs, _ptr(q_out), stream))


def delta_extend_workspace_bytes(shape: delta_shape_t, n_rows: int, max_new: int) -> int:
    n = ctypes.c_size_t(0)
    _check("delta_extend_workspace_bytes",
           delta._lib.delta_extend_workspace_bytes(ctypes.byref(shape), n_rows, max_new, ctypes.byref(n)))
    return n.value


def alloc_extend_workspace(shape, n_rows, max_new, device="cuda") -> torch.Tensor:
    """A workspace (uint8) large enough for delta_extend_attn calls of this shape, with at most so many
    rows and runs of at most max_new."""
    return torch.zeros(delta_extend_workspace_bytes(shape, n_rows, max_new), dtype=torch.uint8, device=device)


def delta_extend_attn(shape, kv: delta_kv_t, q, out, row_offsets, max_new, ws):
    """Causal attention of the new tokens' queries q [rows, n_q_heads, head_dim] over the cache, into
    out.  row_offsets None: one new token per sequence; max_new: at least the longest run."""
    _check_kv(kv, shape)
    _dev("q", q, torch.bfloat16, (None, shape.n_q_heads, shape.head_dim))
    _dev("out", out, torch.bfloat16, tuple(q.shape))
    _offsets(row_offsets, shape.batch)
    _dev("ws", ws)
    stream = _stream_of(kv, q, out, row_offsets, ws)
    _check("delta_extend_attn",
           delta._lib.delta_extend_attn(ctypes.byref(shape), ctypes.byref(kv), q.shape[0], max_new,
                                        _ptr(row_offsets), _ptr(q), _ptr(out), _ptr(ws), _nbytes(ws), stream))


__all__ = ["DeltaError", "delta_rope_t", "delta_rope_append", "delta_extend_workspace_bytes",
           "alloc_extend_workspace", "delta_extend_attn"]
