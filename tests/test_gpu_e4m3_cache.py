"""Decode attention over an e4m3 cache, in all roles, against float64 attention over the values that
the stored bytes stand for."""
import ctypes

import pytest
import torch

from cache_cases import PAGE, Cache, attend, default_scale, queries, worst
from gpu_helpers import D
from oracle import accept as A
from oracle import delta_oracle as O

pytestmark = pytest.mark.gpu


def _full(cache, q, hq, bound=None, sm_scale=0.0):
    d = D()
    kv = cache.on_gpu(d)
    shape = d.make_shape(len(cache.lens), hq, cache.hkv, cache.d, cache.width,
                         bound or max(cache.lens), sm_scale)
    out = torch.full_like(q, float("nan"), device="cuda")
    d.delta_full_attn(shape, kv, q.cuda(), out, d.alloc_workspace(shape))
    torch.cuda.synchronize()
    return out


def _check(cache, q, out, tokens_of, scale=None):
    for b, s in enumerate(cache.lens):
        t = tokens_of(b, s)
        want, tol = attend(q[b], cache.tokens(0, b, t), cache.tokens(1, b, t), scale or default_scale(cache.d))
        assert worst(out[b], want, tol) <= 1, f"sequence {b} of {s} tokens"


@pytest.mark.parametrize("G,hkv,d,scales", [(1, 3, 64, True), (2, 2, 128, False), (3, 1, 64, False),
                                            (4, 8, 128, True), (5, 2, 128, True), (6, 2, 64, True),
                                            (7, 4, 128, True), (8, 1, 128, False), (8, 2, 64, True)])
def test_full_matches_float64(G, hkv, d, scales):
    lens = [1, 15, 16, 17, 100, 129, 1000, 1024]
    cache = Cache(lens, hkv, d, e4m3=True, scales=scales, seed=G * 10 + hkv)
    q = queries(len(lens), G * hkv, d, G)
    _check(cache, q, _full(cache, q, G * hkv), lambda b, s: range(s))


def test_full_of_many_ragged_sequences():
    """More sequences than one lane each, and a bound above every length."""
    lens = [(37 * b * b + 11) % 700 + 1 for b in range(70)]
    cache = Cache(lens, 2, 128, e4m3=True, seed=5, width=80)
    q = queries(len(lens), 14, 128, 6)
    _check(cache, q, _full(cache, q, 14, bound=1280), lambda b, s: range(s))


def test_sharp_and_explicit_softmax_scale():
    cache = Cache([513, 64], 2, 128, e4m3=True, seed=8, k_gain=4.0)
    q = queries(2, 8, 128, 9)
    _check(cache, q, _full(cache, q, 8, sm_scale=0.4), lambda b, s: range(s), scale=0.4)


@pytest.mark.parametrize("d", [64, 128])
def test_every_finite_code_is_read_as_its_value(d):
    """One token: the output is its value.  16 / (d / 16) tokens' worth of codes per sequence, so
    that every one of the 254 finite codes is a value somewhere (NaN codes are not finite inputs)."""
    codes = torch.arange(256, dtype=torch.uint8)
    codes = codes[(codes & 0x7F) != 0x7F]
    codes = torch.cat([codes, codes[:2]])
    B = 256 // d
    cache = Cache([1] * B, 1, d, e4m3=True, scales=False, seed=1)
    for b in range(B):
        v = codes[b * d:(b + 1) * d].view(torch.float8_e4m3fn)
        page = int(cache.table[b, 0])
        cache.stored[1].view(torch.uint8)[page, 0, 0] = v.view(torch.uint8)
        cache.values[1][page, 0, 0] = v.double()
    q = queries(B, 4, d, 2)
    out = _full(cache, q, 4)
    for b in range(B):
        want = cache.tokens(1, b, [0])[0, 0]
        assert torch.equal(out[b].double().cpu(), want.expand(4, d))


def test_every_finite_code_is_read_as_its_key():
    """Two tokens of equal values but for their sign: the output tells the difference of scores,
    q picks one key element at a time."""
    codes = torch.arange(256, dtype=torch.uint8)
    codes = codes[(codes & 0x7F) < 0x70]     # up to 15.0: tanh must not saturate (scale below)
    B = -(-codes.numel() // 8)
    cache = Cache([2] * B, 1, 128, e4m3=True, scales=False, seed=1)
    pick = [[(codes[(8 * b + j) % codes.numel()], 16 * j + (5 * b + j) % 16) for j in range(8)] for b in range(B)]
    q = torch.zeros((B, 8, 128), dtype=torch.bfloat16)
    for b in range(B):
        page = int(cache.table[b, 0])
        k = torch.zeros((2, 128), dtype=torch.uint8)
        for j, (code, at) in enumerate(pick[b]):
            k[0, at] = code
            q[b, j, at] = 1.0
        for which, x in ((0, k.view(torch.float8_e4m3fn)),
                         (1, torch.tensor([1.0, -1.0])[:, None].expand(2, 128).to(torch.float8_e4m3fn))):
            cache.stored[which].view(torch.uint8)[page, 0, :2] = x.contiguous().view(torch.uint8)
            cache.values[which][page, 0, :2] = x.double()
    _check(cache, q, _full(cache, q, 8, sm_scale=0.25), lambda b, s: range(s), scale=0.25)


@pytest.mark.parametrize("unit,agg,path", [(16, 0, 0), (16, 1, 2), (1, 0, 1), (1, 1, 0)])
def test_delta_and_sparse_layers(unit, agg, path):
    """The Delta layer's output is the full layer's, its selection the oracle's up to rounding; the
    sparse layer attends to the device's selection."""
    d = D()
    lens = [1, 40, 200, 777, 1024]
    cache = Cache(lens, 4, 128, e4m3=True, seed=21, k_gain=2.0)
    q = queries(len(lens), 28, 128, 22)
    kv = cache.on_gpu(d)
    shape = d.make_shape(len(lens), 28, 4, 128, cache.width, 1024)
    sel = d.make_select(256, 32, unit, agg, path)
    K, L = 256 // unit, -(-32 // unit)
    ws = d.alloc_workspace(shape, sel)
    idx = torch.full((len(lens), K), -7, dtype=torch.int32, device="cuda")
    cnt = torch.full((len(lens),), -7, dtype=torch.int32, device="cuda")
    phys = torch.full_like(idx, -7)
    out, sparse, direct = (torch.full_like(q, float("nan"), device="cuda") for _ in range(3))
    d.delta_delta_attn_select(shape, kv, q.cuda(), out, sel, idx, cnt, None, ws, sel_phys=phys)
    d.delta_sparse_attn(shape, kv, q.cuda(), sparse, sel, idx, cnt, ws, sel_phys=phys)
    d.delta_sparse_attn(shape, kv, q.cuda(), direct, sel, idx, cnt, ws)
    torch.cuda.synchronize()
    assert torch.equal(out, _full(cache, q, 28))
    assert torch.equal(sparse, direct)
    chosen = []
    for b, s in enumerate(lens):
        k, v = (cache.tokens(w, b, range(s)).numpy() for w in (0, 1))
        _, alpha = O.full_attention(q[b].double().numpy(), k, v, default_scale(128))
        rho, S = O.refresh_units(alpha, unit, K, L, agg)
        got = idx[b, :int(cnt[b])].cpu().numpy()
        assert int(cnt[b]) == min(K, len(S))
        assert A.check_selection(S, K, L, got, rho).ok
        t = (got[:, None] * unit + torch.arange(unit).numpy()).flatten()
        chosen.append(t[t < s])
    _check(cache, q, out, lambda b, s: range(s))
    _check(cache, q, sparse, lambda b, s: chosen[b])


def test_step_of_mixed_caches_with_and_without_workspace():
    """A step whose layers keep bf16 and e4m3 caches: each layer's output is that of its own call."""
    d = D()
    lens = [300, 64, 511]
    roles = [d.DELTA_ROLE_FULL, d.DELTA_ROLE_FULL, d.DELTA_ROLE_DELTA, d.DELTA_ROLE_SPARSE, d.DELTA_ROLE_SPARSE]
    caches = [Cache(lens, 2, 128, e4m3=e, seed=40 + i) for i, e in enumerate([False, True, True, True, False])]
    q = [queries(3, 8, 128, 50 + i).cuda() for i in range(5)]
    kvs = [c.on_gpu(d) for c in caches]
    shape = d.make_shape(3, 8, 2, 128, caches[0].width, 511)
    sel = d.make_select(128, 16)
    ws = d.alloc_workspace(shape, sel)
    got = []
    for step in (d.delta_decode_step, d.delta_decode_step_noalloc):
        outs = [torch.full_like(x, float("nan")) for x in q]
        idx = torch.zeros((1, 3, 8), dtype=torch.int32, device="cuda")
        cnt = torch.zeros((1, 3), dtype=torch.int32, device="cuda")
        step(d.StepArgs(shape, roles, kvs, q, outs, sel, idx, cnt, ws))
        torch.cuda.synchronize()
        got.append((outs, idx, cnt))
    for x, y in zip(got[0][0] + list(got[0][1:]), got[1][0] + list(got[1][1:])):
        assert torch.equal(x, y)
    outs, idx, cnt = got[0]
    for i, c in enumerate(caches):
        def tokens(b, s):
            if i < 3:
                return range(s)
            t = (idx[0, b, :int(cnt[0, b])].cpu()[:, None] * PAGE + torch.arange(PAGE)).flatten()
            return t[t < s]
        _check(c, q[i].cpu(), outs[i], tokens)


def test_refusals():
    d = D()
    c8, c16 = Cache([40], 2, 128, e4m3=True), Cache([40], 2, 128)
    k8, v8 = (x.cuda() for x in c8.stored)
    k16, v16 = (x.cuda() for x in c16.stored)
    table, lens = c8.table.cuda(), torch.tensor([40], dtype=torch.int32, device="cuda")
    one = torch.ones(2, device="cuda")
    with pytest.raises(ValueError, match="k_scale: only caches"):
        d.make_kv(k16, v16, table, lens, k_scale=one)
    with pytest.raises(ValueError, match="v_scale: must be a GPU tensor"):
        d.make_kv(k8, v8, table, lens, v_scale=one.cpu())
    shape = d.make_shape(1, 8, 2, 128, c8.width, 40)
    q = queries(1, 8, 128, 1).cuda()
    ws = d.alloc_workspace(shape)
    out = torch.zeros_like(q)
    for kv, what in ((d.make_kv(k8, v16, table, lens), "v_cache"),
                     (d.make_kv(k16, v8, table, lens), "v_cache"),
                     (d.make_kv(k8, v8, table, lens, k_scale=one[:1]), "k_scale"),
                     (d.make_kv(k8, v8, table, lens, v_scale=one.double()), "v_scale")):
        with pytest.raises(ValueError, match="^" + what):
            d.delta_full_attn(shape, kv, q, out, ws)
    new = torch.zeros((1, 2, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="^k_cache"):
        d.delta_kv_append(shape, k8, v8, table, lens, new, new)
    bad = d.make_kv(k16, v16, table, lens)
    bad.kv_type = 2
    assert d._lib.delta_full_attn(ctypes.byref(shape), ctypes.byref(bad), q.data_ptr(), out.data_ptr(),
                                  ws.data_ptr(), ws.numel(), None) == d.DELTA_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert not out.any()
