"""Host checks of the cache descriptor's element type and scales (no GPU): refused before any launch."""
import ctypes

import pytest
import torch

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


@pytest.mark.parametrize("moved", ["v_cache", "page_table", "seq_lens", "k_scale", "v_scale"])
def test_a_cache_whose_tensors_are_on_two_devices_is_refused(moved, monkeypatch):
    """(The first check, for GPU tensors, is left out: the host's memory and "meta" are two devices.)"""
    monkeypatch.setattr(D, "_dev", lambda name, t, *rest, **kw: t)
    x = dict(k_cache=torch.zeros((3, 2, 16, 64)).to(torch.float8_e4m3fn),
             v_cache=torch.zeros((3, 2, 16, 64)).to(torch.float8_e4m3fn),
             page_table=torch.zeros((1, 3), dtype=torch.int32), seq_lens=torch.zeros(1, dtype=torch.int32),
             k_scale=torch.ones(2), v_scale=torch.ones(2))
    D.make_kv(**x)
    x[moved] = x[moved].to("meta")
    with pytest.raises(ValueError, match=f"^{moved}: on meta"):
        D.make_kv(**x)
