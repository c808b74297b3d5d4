"""A cache descriptor's tensors are checked at every call: one that was resized, transposed or given other
memory in place after make_kv is refused before anything is launched."""
import pytest
import torch

from cache_cases import Cache, queries
from gpu_helpers import D

pytestmark = pytest.mark.gpu


def _shrunk_table(kv):
    kv._tensors[2].resize_(2, 3)


def _shrunk_lengths(kv):
    kv._tensors[3].resize_(1)


def _fewer_rows(kv):
    kv._tensors[0].resize_(kv._tensors[0].shape[0], 2, 8, 64)


def _turned(kv):
    kv._tensors[1].transpose_(2, 3)


def _turned_square(kv):
    kv._tensors[1].transpose_(1, 2)


def _other_memory(kv):
    kv._tensors[0].data = kv._tensors[0].clone()


@pytest.mark.parametrize("change,match", [(_shrunk_table, "^page_table: expected shape"),
                                          (_shrunk_lengths, "^seq_lens: expected shape"),
                                          (_fewer_rows, "^k_cache: expected shape"), (_turned, "^v_cache"),
                                          (_turned_square, "^v_cache: must be contiguous"),
                                          (_other_memory, "^k_cache: its memory")])
@pytest.mark.parametrize("e4m3", [False, True])
def test_a_tensor_changed_in_place_is_refused(change, match, e4m3):
    from paper_2510_09883_amd import extend as E
    d = D()
    hkv = 16 if change is _turned_square else 2    # as many heads as rows of a page
    cache = Cache([40, 60], hkv, 64, e4m3=e4m3, seed=3)
    q = queries(2, 2 * hkv, 64, 4).cuda()
    shape = d.make_shape(2, 2 * hkv, hkv, 64, cache.width, 60)
    kv = cache.on_gpu(d)
    ws, ews = d.alloc_workspace(shape), E.alloc_extend_workspace(shape, 2, 1)
    out = torch.full_like(q, 7.0)
    d.delta_full_attn(shape, kv, q, out, ws)
    torch.cuda.synchronize()
    assert not bool((out == 7.0).all())
    kept = [x for x in kv._tensors[:4]] + [x.data for x in kv._tensors[:4]]   # (what a refused call would read)
    change(kv)
    out.fill_(7.0)
    rows = torch.zeros((2, hkv, 64), dtype=torch.bfloat16, device="cuda")
    for call in (lambda: d.delta_full_attn(shape, kv, q, out, ws),
                 lambda: E.delta_extend_attn(shape, kv, q, out, None, 1, ews),
                 lambda: E.delta_rope_append(shape, kv, q, rows, rows, out)):
        with pytest.raises(ValueError, match=match):
            call()
    torch.cuda.synchronize()
    assert bool((out == 7.0).all()) and len(kept) == 8


@pytest.mark.parametrize("which", [0, 1])
def test_a_scale_changed_in_place_is_refused(which):
    d = D()
    cache = Cache([40, 60], 2, 64, e4m3=True, seed=3)
    q = queries(2, 4, 64, 4).cuda()
    shape = d.make_shape(2, 4, 2, 64, cache.width, 60)
    ws, out = d.alloc_workspace(shape), torch.full_like(q, 7.0)
    name = "kv"[which] + "_scale"
    for change, match in ((lambda s: s.resize_(1), "expected shape"), (lambda s: setattr(s, "data", s.clone()), "its memory")):
        kv = cache.on_gpu(d)
        scale = kv._tensors[4][which][1]
        kept = scale.data
        change(scale)
        with pytest.raises(ValueError, match=f"^{name}: {match}"):
            d.delta_full_attn(shape, kv, q, out, ws)
        assert kept.numel() == 2
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
