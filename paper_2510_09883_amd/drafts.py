"""Python binding of the rounds of drafted tokens of libdelta_attn.so (include/delta_drafts.h): trees of
drafts are laid out, normed, rotated and appended, attended, verified, and what was accepted is kept.
Argument marshalling only, in the manner of the decode-step binding: tensors by device pointer, torch's
current stream, a non-zero status raises DeltaError.  Shapes and cache descriptors come from
delta.make_shape and delta.make_kv.

A run is a tree: its first row is the token decided last, the others are drafts; parents [rows] (int32)
names the place in its run of the row that each one continues, -1: none."""
from __future__ import annotations

import ctypes

import torch

from . import delta
from .delta import DeltaError, _check, _check_kv, _dev, _nbytes, _P, _ptr, _vp
from .delta import delta_kv_t, delta_shape_t
from .extend import _i32, _i64, _offsets, _rows, _stream_of, delta_rope_t

EXPORTED = ["delta_norm_rope_append", "delta_tree_layout", "delta_tree_workspace_bytes", "delta_tree_attn",
            "delta_verify_workspace_bytes", "delta_verify_drafts", "delta_cache_compact"]
DELTA_MOST_DRAFTS = 512
DELTA_NORM_BF16, DELTA_NORM_F32 = 0, 1


class delta_norm_t(ctypes.Structure):
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
                ("weight_type", ctypes.c_int32), ("eps", ctypes.c_float)]


def _bind(lib):
    """Declare the C signatures of include/delta_drafts.h on a loaded library handle."""
    size, shape = ctypes.c_size_t, _P(delta_shape_t)
    lib.delta_norm_rope_append.argtypes = [shape, _P(delta_kv_t), _P(delta_norm_t), _P(delta_rope_t), _i32, _vp,
                                           _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp]
    lib.delta_tree_layout.argtypes = [shape, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _i32, _vp]
    lib.delta_tree_workspace_bytes.argtypes = [shape, _i32, _i32, _P(size)]
    lib.delta_tree_attn.argtypes = [shape, _P(delta_kv_t), _i32, _i32, _vp, _vp, _i32, _vp, _vp, _vp, size, _vp]
    lib.delta_verify_workspace_bytes.argtypes = [_i32, _i32, _P(size)]
    lib.delta_verify_drafts.argtypes = [_i32, _i32, _i32, _vp, _i32, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp,
                                        _vp, _vp, size, _vp]
    lib.delta_cache_compact.argtypes = [shape, _i32, _P(delta_kv_t), _i32, _i32, _vp, _vp, _vp, _vp, _vp]
    for n in EXPORTED:
        getattr(lib, n).restype = ctypes.c_int
    return lib


_bind(delta._lib)   # (calls go to the library that the decode-step binding has loaded)


def delta_norm_rope_append(shape, kv: delta_kv_t, q, k, v, q_out, q_weight=None, k_weight=None, eps=1e-6,
                           inv_freq=None, row_offsets=None, positions=None, interleaved=False):
    """extend.delta_rope_append with the heads of q and k normed first: x * weight / sqrt(mean(x^2) + eps).
    q_weight, k_weight [head_dim], both bfloat16 or both float32 (None: 1)."""
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
    kind = torch.bfloat16
    for w in (q_weight, k_weight):
        if getattr(w, "dtype", None) == torch.float32:
            kind = torch.float32
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None:
            _dev(name, w, kind, (shape.head_dim,))
    norm = delta_norm_t(_ptr(q_weight), _ptr(k_weight),
                        DELTA_NORM_F32 if kind == torch.float32 else DELTA_NORM_BF16, eps)
    rope = None
    if inv_freq is not None:
        _dev("inv_freq", inv_freq, torch.float32, (None,))
        if positions is not None:
            _dev("positions", positions, torch.int32, (n,))
        rope = ctypes.byref(delta_rope_t(inv_freq.data_ptr(), _ptr(positions), 2 * inv_freq.shape[0],
                                         1 if interleaved else 0))
    elif positions is not None:
        raise ValueError("positions: nothing is rotated without inv_freq")
    stream = _stream_of(kv, k, v, q, q_out, q_weight, k_weight, row_offsets, inv_freq, positions)
    _check("delta_norm_rope_append",
           delta._lib.delta_norm_rope_append(ctypes.byref(shape), ctypes.byref(kv), ctypes.byref(norm), rope, n,
                                             _ptr(row_offsets), _ptr(q), qs, k.data_ptr(), ks, v.data_ptr(), vs,
                                             _ptr(q_out), stream))


def delta_tree_layout(shape, seq_lens, parents, positions, masks, row_offsets, max_new):
    """Positions [rows] and masks [rows, words] (int32, bit i of a row: it sees place i of its run) of the
    trees that parents [rows] describes; either output may be None."""
    n = parents.shape[0] if isinstance(parents, torch.Tensor) and parents.dim() else 0
    _dev("parents", parents, torch.int32, (None,))
    _offsets(row_offsets, shape.batch)
    if positions is not None:
        _dev("seq_lens", seq_lens, torch.int32, (shape.batch,))
        _dev("positions", positions, torch.int32, (n,))
    words = 0
    if masks is not None:
        _dev("masks", masks, torch.int32, (n, None))
        words = masks.shape[1]
        if not words:   # (an empty tensor has no address: the library would take it for none)
            raise DeltaError("delta_tree_layout", delta.DELTA_ERR_INVALID_ARG)
    stream = _stream_of(None, parents, seq_lens if positions is not None else None, positions, masks, row_offsets)
    _check("delta_tree_layout",
           delta._lib.delta_tree_layout(ctypes.byref(shape), _ptr(seq_lens) if positions is not None else None, n,
                                        max_new, _ptr(row_offsets), _ptr(parents), _ptr(positions), _ptr(masks), words,
                                        stream))


def delta_tree_workspace_bytes(shape: delta_shape_t, n_rows: int, max_new: int) -> int:
    n = ctypes.c_size_t(0)
    _check("delta_tree_workspace_bytes",
           delta._lib.delta_tree_workspace_bytes(ctypes.byref(shape), n_rows, max_new, ctypes.byref(n)))
    return n.value


def alloc_tree_workspace(shape, n_rows, max_new, device="cuda") -> torch.Tensor:
    """A workspace (uint8) large enough for delta_tree_attn calls of this shape, with at most so many rows
    and runs of at most max_new."""
    return torch.zeros(delta_tree_workspace_bytes(shape, n_rows, max_new), dtype=torch.uint8, device=device)


def delta_tree_attn(shape, kv: delta_kv_t, q, out, masks, row_offsets, max_new, ws):
    """Attention of q [rows, n_q_heads, head_dim] to the tokens before each run and to the rows of the run
    that masks [rows, words] (int32) names, into out.  row_offsets None: one row per sequence; max_new: at
    least the longest run."""
    _check_kv(kv, shape)
    _dev("q", q, torch.bfloat16, (None, shape.n_q_heads, shape.head_dim))
    _dev("out", out, torch.bfloat16, tuple(q.shape))
    _dev("masks", masks, torch.int32, (q.shape[0], None))
    _offsets(row_offsets, shape.batch)
    _dev("ws", ws)
    stream = _stream_of(kv, q, out, masks, row_offsets, ws)
    _check("delta_tree_attn",
           delta._lib.delta_tree_attn(ctypes.byref(shape), ctypes.byref(kv), q.shape[0], max_new, _ptr(row_offsets),
                                      _ptr(masks), masks.shape[1], _ptr(q), _ptr(out), _ptr(ws), _nbytes(ws), stream))


def delta_verify_workspace_bytes(batch: int, vocab: int) -> int:
    n = ctypes.c_size_t(0)
    _check("delta_verify_workspace_bytes", delta._lib.delta_verify_workspace_bytes(batch, vocab, ctypes.byref(n)))
    return n.value


def alloc_verify_workspace(batch, vocab, device="cuda") -> torch.Tensor:
    """A workspace (uint8) large enough for delta_verify_drafts calls of up to so many sequences
    and tokens of the vocabulary."""
    return torch.zeros(delta_verify_workspace_bytes(batch, vocab), dtype=torch.uint8, device=device)


def _probabilities(name, t, rows):
    """A float32 [rows, vocab] GPU tensor whose rows may stand apart; its row stride.  What passes is found out
    first, and what does not is given its message after."""
    if type(t) is torch.Tensor and t.is_cuda and t.dtype == torch.float32:
        have, stride = t.shape, t.stride()
        if len(have) == 2 and stride[1] == 1 and (rows is None or have == rows):
            return stride[0] if have[0] > 1 else have[1]   # (the stride of a single row says nothing)
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a GPU tensor (got device {t.device})")
    if t.dtype != torch.float32:
        raise ValueError(f"{name}: expected {torch.float32}, got {t.dtype}")
    if t.dim() != 2 or (rows is not None and tuple(t.shape) != rows):
        raise ValueError(f"{name}: expected shape {rows or (None, None)}, got {tuple(t.shape)}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the values of a row must lie one behind the other")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def delta_verify_drafts(target, draft, tokens, parents, uniform, row_offsets, path, n_path, next_token, ws):
    """Which drafts stand: path [batch, max_new] gets the places of the accepted rows (-1 behind them), n_path
    [batch] their count, next_token [batch] the token after them.  target [rows, vocab] and draft (the same,
    or None: the drafts were not drawn) are float32 probabilities, tokens and parents [rows] int32, uniform
    [rows] float32."""
    ts = _probabilities("target", target, None)
    rows, vocab = target.shape
    ds = 0 if draft is None else _probabilities("draft", draft, (rows, vocab))
    _dev("tokens", tokens, torch.int32, (rows,))
    _dev("parents", parents, torch.int32, (rows,))
    _dev("uniform", uniform, torch.float32, (rows,))
    _dev("path", path, torch.int32, (None, None))
    batch = path.shape[0]
    _dev("n_path", n_path, torch.int32, (batch,))
    _dev("next_token", next_token, torch.int32, (batch,))
    _offsets(row_offsets, batch)
    _dev("ws", ws)
    stream = _stream_of(None, target, draft, tokens, parents, uniform, row_offsets, path, n_path, next_token, ws)
    _check("delta_verify_drafts",
           delta._lib.delta_verify_drafts(batch, rows, path.shape[1], _ptr(row_offsets), vocab, _ptr(target), ts,
                                          _ptr(draft), ds, _ptr(tokens), _ptr(parents), _ptr(uniform), _ptr(path),
                                          _ptr(n_path), _ptr(next_token), _ptr(ws), _nbytes(ws), stream))


class CacheStack:
    """The cache descriptors of a model's layers, for calls that work on all of them at once: built once, reused
    every round.  All share seq_lens.  As with a single descriptor, every call looks whether the tensors are
    still what make_kv was given."""

    def __init__(self, shape, kvs):
        if not kvs:
            raise ValueError("a stack needs at least one layer")
        for kv in kvs:
            _check_kv(kv, shape)
            mine, first = getattr(kv, "_tensors", None), getattr(kvs[0], "_tensors", None)
            if mine and first and mine[0].device != first[0].device:
                raise ValueError(f"a layer's cache is on {mine[0].device}, the first one's on {first[0].device}")
        self.shape, self.n, self.layers = shape, len(kvs), list(kvs)
        self.kvs = (delta_kv_t * self.n)(*kvs)
        self._sizes = _sizes(shape)
        # every tensor once, as tables and lengths are often those of all layers (scales are not read)
        made = {id(x): (x, *m) for kv in kvs if hasattr(kv, "_tensors") for x, m in zip(kv._tensors, kv._made)}
        self._tensors, self._shapes, self._places = map(list, zip(*made.values())) if made else ([], [], [])

    def _check(self):
        """All tensors at once (28 layers: 11 us; one descriptor after the other 31); what has changed finds
        its message after."""
        one = torch.Tensor
        if (self._sizes != _sizes(self.shape) or list(map(one.data_ptr, self._tensors)) != self._places
                or list(map(one.size, self._tensors)) != self._shapes
                or False in map(one.is_contiguous, self._tensors)):
            for kv in self.layers:
                _check_kv(kv, self.shape)


def _sizes(shape):
    return shape.n_kv_heads, shape.page_size, shape.head_dim, shape.batch, shape.max_pages_per_seq


def delta_cache_compact(stack: CacheStack, n_rows, row_offsets, path, n_path, new_lens=None):
    """Moves the accepted rows path [batch, max_new], n_path [batch] of every run together in the caches of
    all layers; new_lens [batch] (None: not written) gets the lengths, and may be the layers' seq_lens."""
    shape = stack.shape
    stack._check()
    _dev("path", path, torch.int32, (shape.batch, None))
    _dev("n_path", n_path, torch.int32, (shape.batch,))
    if new_lens is not None:
        _dev("new_lens", new_lens, torch.int32, (shape.batch,))
    _offsets(row_offsets, shape.batch)
    stream = _stream_of(stack.layers[0], row_offsets, path, n_path, new_lens)
    _check("delta_cache_compact",
           delta._lib.delta_cache_compact(ctypes.byref(shape), stack.n, stack.kvs, n_rows, path.shape[1],
                                          _ptr(row_offsets), _ptr(path), _ptr(n_path), _ptr(new_lens), stream))


__all__ = ["DeltaError", "delta_norm_t", "delta_norm_rope_append", "delta_tree_layout", "delta_tree_workspace_bytes",
           "alloc_tree_workspace", "delta_tree_attn", "delta_verify_workspace_bytes", "alloc_verify_workspace",
           "delta_verify_drafts", "CacheStack", "delta_cache_compact"]
