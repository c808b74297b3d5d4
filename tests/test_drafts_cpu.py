"""Host checks of include/delta_drafts.h: exports, argument refusals and workspace sizes (no GPU)."""
import ctypes
import os
import re

import pytest

from paper_2510_09883_amd import delta as D
from paper_2510_09883_amd import drafts as T
from paper_2510_09883_amd import extend as E

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "delta_drafts.h")
FAKE = ctypes.c_void_p(0x1000)


def shape(**kw):
    s = dict(batch=4, n_q_heads=8, n_kv_heads=2, head_dim=128, max_pages_per_seq=64, max_seq_len=1024)
    s.update(kw)
    return D.make_shape(**s)


def cache(k=0x1000, v=0x2000, table=0x1000, lens=0x1000, n_pages=0, kv_type=0):
    return D.delta_kv_t(k, v, table, lens, n_pages, kv_type)


def test_library_exports_the_header():
    text = open(HEADER).read()
    names = sorted(set(re.findall(r"^int (delta_\w+)\s*\(", text, re.M)))
    assert names == sorted(T.EXPORTED)
    lib = ctypes.CDLL(D.LIB_PATH)
    assert all(hasattr(lib, n) for n in names)
    assert f"#define DELTA_MOST_DRAFTS {T.DELTA_MOST_DRAFTS}" in text


def append(s=None, kv=None, norm=(None, None, 0, 1e-6), rope=None, n_rows=4, offsets=FAKE, q=FAKE, qs=1024, k=FAKE,
           ks=256, v=FAKE, vs=256, q_out=FAKE):
    norm = ctypes.byref(T.delta_norm_t(*norm)) if norm else None
    return D._lib.delta_norm_rope_append(ctypes.byref(s or shape()), ctypes.byref(kv or cache()), norm,
                                         ctypes.byref(rope) if rope else None, n_rows, offsets, q, qs, k, ks, v, vs,
                                         q_out, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(norm=None), -1), (dict(norm=(None, None, 2, 1e-6)), -1), (dict(norm=(None, None, 0, -1e-6)), -1),
    (dict(norm=(None, None, 0, float("nan"))), -1), (dict(norm=(None, None, 0, float("inf"))), -1),
    (dict(norm=(0x1008, None, 0, 0.0)), -1), (dict(norm=(None, 0x1004, 1, 0.0)), -1),
    (dict(s=shape(head_dim=96)), -2), (dict(n_rows=-1), -1), (dict(offsets=None, n_rows=5), -1), (dict(k=None), -1),
    (dict(q=None), -1), (dict(qs=1016), -1), (dict(ks=260), -1), (dict(vs=0), -1), (dict(q_out=ctypes.c_void_p(0x1002)), -1),
    (dict(rope=E.delta_rope_t(None, None, 128, 0)), -1), (dict(rope=E.delta_rope_t(0x1000, None, 24, 0)), -1),
    (dict(n_rows=1 << 26), -2), (dict(qs=1536), -1), (dict(kv=cache(lens=None)), -1),
    (dict(n_rows=0, k=None, v=None, q=None, q_out=None), 0),
])
def test_append_arguments(kw, rc):
    assert append(**kw) == rc


def layout(s=None, lens=FAKE, n_rows=9, max_new=4, offsets=FAKE, parents=FAKE, positions=FAKE, masks=FAKE, words=1):
    return D._lib.delta_tree_layout(ctypes.byref(s or shape()), lens, n_rows, max_new, offsets, parents, positions, masks,
                                    words, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(s=shape(batch=0)), -1), (dict(n_rows=-1), -1), (dict(max_new=-1), -1), (dict(max_new=10), -1),
    (dict(offsets=None), -1), (dict(offsets=None, n_rows=4, max_new=0), -1), (dict(parents=None), -1), (dict(lens=None), -1),
    (dict(positions=None, masks=None), -1), (dict(words=0), -1), (dict(n_rows=100, max_new=33), -1),
    (dict(n_rows=600, max_new=513, words=20), -2), (dict(n_rows=1 << 24), -2), (dict(s=shape(batch=65536)), -2),
    (dict(n_rows=0, max_new=0, parents=None), 0), (dict(max_new=0), 0),
])
def test_layout_arguments(kw, rc):
    assert layout(**kw) == rc


def attend(s=None, kv=None, n_rows=4, max_new=1, offsets=FAKE, masks=FAKE, words=1, q=FAKE, out=FAKE, ws=FAKE,
           ws_bytes=1 << 40):
    return D._lib.delta_tree_attn(ctypes.byref(s or shape()), ctypes.byref(kv or cache()), n_rows, max_new, offsets, masks,
                                  words, q, out, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(s=shape(page_size=32)), -2), (dict(n_rows=-1), -1), (dict(max_new=-1), -1), (dict(max_new=5), -1),
    (dict(offsets=None, n_rows=3), -1), (dict(offsets=None, max_new=0), -1), (dict(q=None), -1), (dict(out=None), -1),
    (dict(masks=None), -1), (dict(words=0), -1), (dict(n_rows=40, max_new=33), -1), (dict(ws=None), -1),
    (dict(ws_bytes=8), -3), (dict(ws=ctypes.c_void_p(0x1010)), -1), (dict(q=ctypes.c_void_p(0x1004)), -1),
    (dict(n_rows=1 << 26, max_new=4), -2), (dict(n_rows=600, max_new=513, words=17), -2), (dict(kv=cache(kv_type=3)), -1),
    (dict(s=shape(max_seq_len=(1 << 31) - 400, max_pages_per_seq=1 << 27)), -2),
    (dict(n_rows=0, max_new=0), 0), (dict(max_new=0), 0),
])
def test_attention_arguments(kw, rc):
    assert attend(**kw) == rc


def test_a_workspace_of_the_largest_call_serves_smaller_ones():
    """The library accepts it: a call of null queries gets past the workspace check and is refused after it."""
    for batch, held in ((1, 131072), (4, 1024), (64, 20000), (300, 512)):
        s = shape(batch=batch, max_pages_per_seq=8192, max_seq_len=held)
        most = T.delta_tree_workspace_bytes(s, 9000, 512)
        assert most % 256 == 0
        for n in (1, 2, 7, 40, 64, 300, 500, 1000, 4096, 9000):
            for m in sorted({1, 2, 8, 9, 16, 17, 33, 65, min(n, 512)}):
                if m <= n:
                    own = T.delta_tree_workspace_bytes(s, n, m)
                    assert own <= most
                    assert attend(s=s, n_rows=n, max_new=m, q=None, words=16, ws_bytes=own) == -1


def verify(batch=2, n_rows=5, max_new=3, offsets=FAKE, vocab=40, target=FAKE, ts=40, draft=FAKE, ds=40, tokens=FAKE,
           parents=FAKE, uniform=FAKE, path=FAKE, n_path=FAKE, nxt=FAKE, ws=FAKE, ws_bytes=1 << 30):
    return D._lib.delta_verify_drafts(batch, n_rows, max_new, offsets, vocab, target, ts, draft, ds, tokens, parents,
                                      uniform, path, n_path, nxt, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(batch=0), -1), (dict(n_rows=-1), -1), (dict(max_new=0), -1), (dict(max_new=6), -1), (dict(offsets=None), -1),
    (dict(vocab=0), -1), (dict(ts=39), -1), (dict(ds=39), -1), (dict(target=None), -1), (dict(tokens=None), -1),
    (dict(parents=None), -1), (dict(uniform=None), -1), (dict(path=None), -1), (dict(n_path=None), -1), (dict(nxt=None), -1),
    (dict(ws=None), -1), (dict(ws=ctypes.c_void_p(0x1010)), -1), (dict(ws_bytes=100), -3), (dict(batch=65536), -2),
    (dict(vocab=(1 << 20) + 1, ts=1 << 21, ds=1 << 21), -2), (dict(n_rows=600, max_new=513), -2),
    (dict(n_rows=1 << 24), -2),
])
def test_verification_arguments(kw, rc):
    assert verify(**kw) == rc


def test_verification_workspace():
    assert T.delta_verify_workspace_bytes(1, 1) <= T.delta_verify_workspace_bytes(8, 1 << 20)
    for bad in ((0, 5), (5, 0), (65536, 5), (5, (1 << 20) + 1)):
        with pytest.raises(D.DeltaError):
            T.delta_verify_workspace_bytes(*bad)


def compact(s=None, kvs=None, n_layers=None, n_rows=9, max_new=4, offsets=FAKE, path=FAKE, n_path=FAKE, lens=None):
    kvs = kvs or [cache(), cache(0x3000, 0x4000, kv_type=1)]
    arr = (D.delta_kv_t * len(kvs))(*kvs)
    return D._lib.delta_cache_compact(ctypes.byref(s or shape()), len(kvs) if n_layers is None else n_layers, arr, n_rows,
                                      max_new, offsets, path, n_path, lens, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(n_layers=0), -1), (dict(kvs=[cache(), cache(0x3000, 0x4000, lens=0x2000)]), -1), (dict(kvs=[cache(k=0x1008)]), -1),
    (dict(kvs=[cache(), cache(0x3000, None)]), -1), (dict(kvs=[cache(v=0x1000)]), -1), (dict(kvs=[cache(), cache(0x3000)]), -1),
    (dict(kvs=[cache(), cache(0x2000, 0x3000)]), -1), (dict(n_rows=-1), -1), (dict(max_new=0), -1), (dict(max_new=10), -1),
    (dict(offsets=None), -1), (dict(path=None), -1), (dict(n_path=None), -1), (dict(s=shape(head_dim=80)), -2),
    (dict(n_rows=600, max_new=513), -2),
])
def test_compaction_arguments(kw, rc):
    assert compact(**kw) == rc
