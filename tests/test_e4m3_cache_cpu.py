"""Host checks of the cache descriptor's element type and scales (no GPU): refused before any launch."""
import ctypes

import pytest

from paper_2510_09883_amd import delta as D


@pytest.mark.parametrize("kv_type,k_scale,v_scale", [(2, None, None), (-1, None, None),
                                                     (0, 0x1000, None), (0, None, 0x1000)])
def test_kv_type_and_scales_are_checked(kv_type, k_scale, v_scale):
    shape = D.make_shape(2, 8, 2, 128, 16, 256)
    kv = D.delta_kv_t(0x1000, 0x1000, 0x1000, 0x1000, 0, kv_type, k_scale, v_scale)
    fake = ctypes.c_void_p(0x1000)
    need = D.delta_workspace_bytes(shape)
    rc = D._lib.delta_full_attn(ctypes.byref(shape), ctypes.byref(kv), fake, fake, fake, need, None)
    assert rc == D.DELTA_ERR_INVALID_ARG


@pytest.mark.parametrize("k,v", [(0x1001, 0x1000), (0x1000, 0x1008)])
def test_an_e4m3_cache_that_is_not_aligned_is_refused(k, v):
    shape = D.make_shape(2, 8, 2, 128, 16, 256)
    kv = D.delta_kv_t(k, v, 0x1000, 0x1000, 0, D.DELTA_KV_E4M3)
    fake = ctypes.c_void_p(0x1000)
    need = D.delta_workspace_bytes(shape)
    rc = D._lib.delta_full_attn(ctypes.byref(shape), ctypes.byref(kv), fake, fake, fake, need, None)
    assert rc == D.DELTA_ERR_INVALID_ARG


def test_a_descriptor_of_five_fields_is_a_bf16_cache():
    kv = D.delta_kv_t(1, 2, 3, 4, 5)
    assert (kv.kv_type, kv.k_scale, kv.v_scale) == (D.DELTA_KV_BF16, None, None)
