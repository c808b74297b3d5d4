"""Host checks of include/delta_extend.h: exports, argument refusals and workspace sizes (no GPU)."""
import ctypes
import os
import re

import pytest

from paper_2510_09883_amd import delta as D
from paper_2510_09883_amd import extend as E

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "delta_extend.h")
FAKE = ctypes.c_void_p(0x1000)


def shape(**kw):
    s = dict(batch=4, n_q_heads=8, n_kv_heads=2, head_dim=128, max_pages_per_seq=64, max_seq_len=1024)
    s.update(kw)
    return D.make_shape(**s)


def test_library_exports_the_header():
    names = sorted(set(re.findall(r"^int (delta_\w+)\s*\(", open(HEADER).read(), re.M)))
    assert names == sorted(E.EXPORTED)
    lib = ctypes.CDLL(D.LIB_PATH)
    assert all(hasattr(lib, n) for n in names)


def append(s=None, kv=None, rope=None, n_rows=4, offsets=FAKE, q=FAKE, qs=1024, k=FAKE, ks=256, v=FAKE, vs=256,
           q_out=FAKE):
    kv = kv or D.delta_kv_t(0x1000, 0x1000, 0x1000, 0x1000, 0)
    return D._lib.delta_rope_append(ctypes.byref(s or shape()), ctypes.byref(kv), ctypes.byref(rope) if rope else None,
                                    n_rows, offsets, q, qs, k, ks, v, vs, q_out, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(s=shape(head_dim=96)), -2), (dict(s=shape(n_q_heads=7)), -1), (dict(n_rows=-1), -1),
    (dict(offsets=None, n_rows=5), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(q=None), -1),
    (dict(q_out=None), -1), (dict(qs=1023), -1), (dict(qs=1016), -1), (dict(ks=255), -1), (dict(ks=260), -1),
    (dict(vs=0), -1), (dict(k=ctypes.c_void_p(0x1008)), -1), (dict(q_out=ctypes.c_void_p(0x1002)), -1),
    (dict(rope=E.delta_rope_t(None, None, 128, 0)), -1), (dict(rope=E.delta_rope_t(0x1000, None, 0, 0)), -1),
    (dict(rope=E.delta_rope_t(0x1000, None, 24, 0)), -1), (dict(rope=E.delta_rope_t(0x1000, None, 144, 0)), -1),
    (dict(rope=E.delta_rope_t(0x1000, None, 64, 2)), -1), (dict(n_rows=1 << 26), -2),
    (dict(kv=D.delta_kv_t(0x1008, 0x1000, 0x1000, 0x1000, 0)), -1),
    (dict(kv=D.delta_kv_t(0x1000, 0x1000, None, 0x1000, 0)), -1),
    (dict(kv=D.delta_kv_t(0x1000, 0x1000, 0x1000, 0x1000, 0, 3)), -1),
    (dict(n_rows=0, k=None, v=None, q=None, q_out=None), 0),
])
def test_append_arguments(kw, rc):
    assert append(**kw) == rc


def test_append_refuses_more_rows_than_a_launch_has_workgroups():
    small = shape(batch=1, n_q_heads=1, n_kv_heads=1, head_dim=64)
    assert append(small, n_rows=1 << 24, qs=64, ks=64, vs=64) == -2


def extend(s=None, n_rows=4, max_new=1, offsets=FAKE, q=FAKE, out=FAKE, ws=FAKE, ws_bytes=1 << 40):
    kv = D.delta_kv_t(0x1000, 0x1000, 0x1000, 0x1000, 0)
    return D._lib.delta_extend_attn(ctypes.byref(s or shape()), ctypes.byref(kv), n_rows, max_new, offsets, q, out,
                                    ws, ws_bytes, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(s=shape(page_size=32)), -2), (dict(n_rows=-1), -1), (dict(max_new=-1), -1), (dict(max_new=5), -1),
    (dict(offsets=None, n_rows=3), -1), (dict(offsets=None, max_new=0), -1), (dict(q=None), -1), (dict(out=None), -1),
    (dict(ws=None), -1), (dict(ws_bytes=8), -3), (dict(ws=ctypes.c_void_p(0x1010)), -1),
    (dict(q=ctypes.c_void_p(0x1004)), -1), (dict(n_rows=1 << 26, max_new=4), -2),
    (dict(n_rows=0, max_new=0), 0), (dict(max_new=0), 0),
])
def test_extend_arguments(kw, rc):
    assert extend(**kw) == rc


def test_workspace_grows_with_the_rows_alone():
    """One sized for the most rows serves every smaller call, whatever its runs and lengths: the library
    accepts it (a call of null queries gets past the workspace check and is refused after it)."""
    part = 4 * (128 + 2)
    for batch, held in ((1, 131072), (4, 1024), (64, 20000), (300, 64)):
        s = shape(batch=batch, max_pages_per_seq=8192, max_seq_len=held)
        sizes = [E.delta_extend_workspace_bytes(s, n, min(n, m)) for n, m in ((1, 1), (5, 3), (700, 700), (9000, 9000))]
        assert sizes == sorted(sizes) and all(x % 256 == 0 for x in sizes)
        assert sizes[-1] <= 131072 * (part + 4) + 2048
        for n in (1, 2, 7, 40, 64, 300, 500, 1000, 4096, 9000):
            for m in sorted({1, 2, 9, n // 2, n} - {0}):
                if m <= n:
                    assert extend(s=s, n_rows=n, max_new=m, q=None, ws_bytes=sizes[-1]) == -1
                    assert extend(s=s, n_rows=n, max_new=m, q=None,
                                  ws_bytes=E.delta_extend_workspace_bytes(s, n, m)) == -1
    with pytest.raises(D.DeltaError):
        E.delta_extend_workspace_bytes(shape(n_kv_heads=1, n_q_heads=16), 1, 1)


@pytest.mark.parametrize("batch,held,larger,smaller", [(16384, 128, (327680, 20), (262144, 16)),
                                                       (20000, 64, (640000, 32), (320000, 16))])
def test_a_call_smaller_than_one_that_is_taken_is_taken(batch, held, larger, smaller):
    """More than 65535 tiles of 32 rows: the call goes to the kernel of larger tiles."""
    s = shape(batch=batch, n_q_heads=8, n_kv_heads=1, max_pages_per_seq=-(-held // 16), max_seq_len=held)
    size = E.delta_extend_workspace_bytes(s, *larger)
    assert E.delta_extend_workspace_bytes(s, *smaller) <= size
    for n_rows, max_new in (larger, smaller):
        assert extend(s=s, n_rows=n_rows, max_new=max_new, q=None, ws_bytes=size) == -1   # (null queries)


def test_more_tiles_than_a_launch_has_are_refused():
    """2^21 rows of 8 query heads per KV head are 65536 tiles of 256 rows."""
    s = shape(batch=1, n_q_heads=8, n_kv_heads=1, max_pages_per_seq=1 << 17, max_seq_len=1 << 21)
    assert extend(s=s, n_rows=1 << 21, max_new=1 << 21, q=None) == -2
    assert extend(s=s, n_rows=(1 << 21) - 512, max_new=(1 << 21) - 512, q=None) == -1
    with pytest.raises(D.DeltaError):
        E.delta_extend_workspace_bytes(s, 1 << 21, 1 << 21)


def test_rotation_in_place_of_rows_that_stand_apart_is_refused():
    """q_out's rows lie one behind the other: over such a q they would fall on rows still to be read."""
    assert append(qs=1536) == -1
