"""Decode attention over e4m3 caches where a workgroup's piece is long (blocks of four pages a wave, a second
listing, a second chunk of staged logits, a last single page), and sparse layers at head size 64."""
import pytest
import torch

from cache_cases import Cache, attend, default_scale, queries, worst
from gpu_helpers import D
from oracle import accept as A
from oracle import delta_oracle as O

pytestmark = pytest.mark.gpu


def _layers(cache, q, hq, budget, unit, bound):
    """Outputs of a full, a Delta and a sparse layer, and the selection."""
    d = D()
    B, recent = len(cache.lens), 32
    kv = cache.on_gpu(d)
    shape = d.make_shape(B, hq, cache.hkv, cache.d, cache.width, bound)
    sel = d.make_select(budget, recent, unit)
    ws = d.alloc_workspace(shape, sel)
    idx = torch.full((B, budget // unit), -7, dtype=torch.int32, device="cuda")
    cnt = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    full, delta, sparse = (torch.full_like(q, float("nan"), device="cuda") for _ in range(3))
    qg = q.cuda()
    d.delta_full_attn(shape, kv, qg, full, ws)
    d.delta_delta_attn_select(shape, kv, qg, delta, sel, idx, cnt, None, ws)
    d.delta_sparse_attn(shape, kv, qg, sparse, sel, idx, cnt, ws)
    torch.cuda.synchronize()
    assert torch.equal(full, delta)
    assert not bool(full.isnan().any()) and not bool(sparse.isnan().any())
    return full.cpu(), sparse.cpu(), idx.cpu(), cnt.cpu()


def _check(cache, q, result, budget, unit, seqs):
    full, sparse, idx, cnt = result
    scale = default_scale(cache.d)
    K, L = budget // unit, -(-32 // unit)
    for b in seqs:
        s = cache.lens[b]
        k, v = (cache.tokens(w, b, range(s)) for w in (0, 1))
        want, tol = attend(q[b], k, v, scale)
        assert worst(full[b], want, tol) <= 1, f"full layer, sequence {b} of {s} tokens"
        _, alpha = O.full_attention(q[b].double().numpy(), k.numpy(), v.numpy(), scale)
        rho, S = O.refresh_units(alpha, unit, K, L)
        got = idx[b, :int(cnt[b])].numpy()
        verdict = A.check_selection(S, K, L, got, rho)
        assert verdict.ok, (b, verdict.reasons)
        t = torch.from_numpy((got[:, None] * unit + torch.arange(unit).numpy()).flatten())
        t = t[t < s].long()
        want, tol = attend(q[b], k[t], v[t], scale)
        assert worst(sparse[b], want, tol) <= 1, f"sparse layer, sequence {b} of {s} tokens"


@pytest.mark.parametrize("G,d", [(7, 128), (8, 128), (8, 64), (3, 64), (1, 128)])
def test_one_piece_a_pair(G, d):
    """256 pairs: every sequence is one workgroup's.  17000 tokens are 1063 pages, more than are listed at
    once, and several chunks of logits; 4993 an odd number of pages, the last of one token; 3584 and
    3585 tokens end with a chunk of 224 pages and one page after it, 4096 and 4097 with one of 256."""
    lens = [17000, 4993, 3584, 3585, 4096, 4097, 2047] + [(29 * b) % 70 + 1 for b in range(249)]
    cache = Cache(lens, 1, d, e4m3=True, seed=G + d)
    q = queries(256, G, d, G)
    _check(cache, q, _layers(cache, q, G, 1024, 16, 17000), 1024, 16, [*range(10), 100, 255])


@pytest.mark.parametrize("G,d", [(8, 64), (5, 128)])
def test_balanced_runs_of_long_pieces(G, d):
    """16 ragged sequences with 8 KV heads: runs of about 150 pages that span pairs."""
    lens = [4000 + (977 * b) % 900 for b in range(15)] + [33]
    cache = Cache(lens, 8, d, e4m3=True, seed=G)
    q = queries(16, 8 * G, d, G)
    _check(cache, q, _layers(cache, q, 8 * G, 1024, 16, max(lens)), 1024, 16, [0, 1, 7, 14, 15])


@pytest.mark.parametrize("unit", [16, 1])
@pytest.mark.parametrize("G,hkv", [(3, 2), (8, 1), (4, 4), (1, 3)])
def test_sparse_layers_of_small_heads(G, hkv, unit):
    """Head size 64, pages and single tokens, selections that fill a tile and that do not."""
    lens = [1, 17, 40, 255, 777, 1500, 3001]
    cache = Cache(lens, hkv, 64, e4m3=True, seed=10 * G + unit, k_gain=2.0)
    q = queries(len(lens), G * hkv, 64, G)
    for budget in (256, 48):
        _check(cache, q, _layers(cache, q, G * hkv, budget, unit, 3001), budget, unit, range(len(lens)))


@pytest.mark.parametrize("unit,d", [(16, 128), (1, 128), (1, 64)])
def test_long_selections(unit, d):
    """Sparse walks of many pages and of many single tokens in one piece."""
    lens = [7000, 6500] + [(31 * b) % 90 + 1 for b in range(254)]
    cache = Cache(lens, 1, d, e4m3=True, seed=unit + d)
    q = queries(256, 4, d, 5)
    _check(cache, q, _layers(cache, q, 4, 4096, unit, 7000), 4096, unit, [0, 1, 2, 200])
