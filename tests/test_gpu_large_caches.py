"""Caches whose element offsets pass 32 bits: append, attention of new tokens and a decode layer on pages at
both ends of more than 2^32 elements."""
import pytest
import torch

from cache_cases import PAGE, attend, default_scale, worst
from gpu_helpers import D

pytestmark = pytest.mark.gpu

HQ, HKV, HD, PAGES = 16, 8, 128, 262144 + 40     # 2^32 elements are 262144 pages


@pytest.mark.parametrize("e4m3", [False, True])
def test_pages_past_32_bits(e4m3):
    from paper_2510_09883_amd import extend as E
    d = D()
    kind = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    k, v = (torch.empty((PAGES, HKV, PAGE, HD), dtype=kind, device="cuda") for _ in range(2))
    table = torch.tensor([[PAGES - 1, 7, 262144, PAGES - 3, 131072]], dtype=torch.int32)
    n = 75
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    kv = d.make_kv(k, v, table.cuda(), lens)
    shape = d.make_shape(1, HQ, HKV, HD, table.shape[1], n)
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((n, HQ + 2 * HKV, HD), generator=g).to(torch.bfloat16)
    dev = qkv.cuda()
    off = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    q, out = (torch.zeros((n, HQ, HD), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    E.delta_rope_append(shape, kv, dev[:, :HQ], dev[:, HQ:HQ + HKV], dev[:, HQ + HKV:], q, row_offsets=off)
    E.delta_extend_attn(shape, kv, q, out, off, n, E.alloc_extend_workspace(shape, n, n))
    last = torch.zeros((1, HQ, HD), dtype=torch.bfloat16, device="cuda")
    d.delta_full_attn(shape, kv, q[n - 1:].contiguous(), last, d.alloc_workspace(shape))
    torch.cuda.synchronize()
    assert torch.equal(q.cpu(), qkv[:, :HQ])    # nothing is rotated
    held = [x.float().to(kind).double() for x in (qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:])]
    for cache, want in zip((k, v), held):
        t = torch.arange(n)
        page = table[0, t // PAGE].long().cuda()
        got = cache.view(torch.uint8 if e4m3 else torch.int16)[page, :, (t % PAGE).cuda()].view(kind)
        assert torch.equal(got.cpu().double(), want)
    for j in (0, 20, 50, n - 1):
        want, tol = attend(qkv[j, :HQ], held[0][:j + 1], held[1][:j + 1], default_scale(HD), 2.0 ** -8)
        assert worst(out[j], want, tol) <= 1
    want, tol = attend(qkv[n - 1, :HQ], held[0], held[1], default_scale(HD))
    assert worst(last[0], want, tol) <= 1
