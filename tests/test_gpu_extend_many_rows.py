"""delta_extend_attn's kernel of 256-row tiles against float64: both head sizes and cache types, every kind
of group, several sequences, tiles of few rows, pieces and their join, rows that see nothing, infinite
and NaN values, and its captured form."""
import pytest
import torch

from cache_cases import Cache, attend, default_scale, queries, worst
from gpu_helpers import D
from many_row_cases import HIDDEN, MANY_ROWS, MOST_TILES
from test_gpu_extend_attn import Call, E, P_ROUND

pytestmark = pytest.mark.gpu


def picks(n, G, seed):
    """The run's ends, tokens around the first, a middle and the last border of tiles, and some others."""
    g = torch.Generator().manual_seed(seed)
    at = {0, n - 1, *torch.randint(0, n, (16,), generator=g).tolist()}
    tiles = n * G // 256
    for t in {1, tiles // 2, tiles}:
        at |= {256 * t // G + i for i in (-1, 0, 1)}
    return sorted(j for j in at if 0 <= j < n)


def check(c, seed=0):
    torch.cuda.synchronize()
    out, row, G = c.out.cpu(), 0, c.hq // c.cache.hkv
    for b, (s, n) in enumerate(zip(c.lens, c.new)):
        for j in picks(n, G, seed + b) if n else ():
            t = range(max(0, s - n + j + 1))
            want, tol = attend(c.q[row + j], c.cache.tokens(0, b, t), c.cache.tokens(1, b, t), c.scale, P_ROUND)
            assert worst(out[row + j], want, tol) <= 1, f"row {j} of run {b} ({n} of {s} tokens)"
        if s < n:
            assert not out[row:row + n - s].any()
        row += n
    assert not bool(out[:row].isnan().any())
    assert bool((out[row:] == 7.0).all()), "rows behind the last run were written"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("case", MANY_ROWS)
def test_many_rows(case, e4m3, d):
    lens, new, hq, hkv = case
    c = Call(list(lens), list(new), hq, hkv, d, e4m3=e4m3, seed=d + hq, pad=3)
    c.run()
    check(c)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("at", [200, 255, 640, 1023, 1024, 1498])
def test_values_of_tokens_that_a_row_does_not_see(at, e4m3, d):
    """Token `at` has an infinite (e4m3: NaN) value element, the token after it a key of NaN."""
    lens, new, hq, hkv = HIDDEN
    c = Call(list(lens), list(new), hq, hkv, d, e4m3=e4m3, seed=at)
    k, v = c.kv._tensors[:2]
    raw_k, raw_v = (x.view(torch.uint8 if e4m3 else torch.int16) for x in (k, v))
    place = lambda t: (int(c.cache.table[0, t // 16]), slice(None), t % 16)   # noqa: E731
    raw_v[place(at)][:, 5] = 0x7F if e4m3 else 0x7F80
    raw_k[place(at + 1)] = 0x7F if e4m3 else 0x7FC0
    c.run()
    torch.cuda.synchronize()
    out, held, n = c.out.cpu(), lens[0], new[0]
    first = held - n     # the token of the first row
    for last in sorted({first, at - 60, at - 51, at - 1, at, at + 1, at + 40, held - 1, *range(first, held, 97)}):
        if not first <= last < held:
            continue
        got = out[last - first].clone()
        if last > at:
            assert bool(got.isnan().all()), last     # it sees the key of NaN
            continue
        t = range(last + 1)
        want, tol = attend(c.q[last - first], c.cache.tokens(0, 0, t), c.cache.tokens(1, 0, t), c.scale, P_ROUND)
        if last == at:
            assert not bool(got[:, 5].isfinite().any())
            got[:, 5] = want[:, 5].to(got.dtype)
        assert worst(got, want, tol) <= 1, last
    for j in range(new[1]):
        t = range(lens[1] - new[1] + j + 1)
        want, tol = attend(c.q[n + j], c.cache.tokens(0, 1, t), c.cache.tokens(1, 1, t), c.scale, P_ROUND)
        assert worst(out[n + j], want, tol) <= 1


@pytest.mark.parametrize("e4m3", [False, True])
def test_sharp_scores_a_larger_bound_and_replays(e4m3):
    """A bound of the runs and of the lengths above both, scores that one token decides; captured once, with
    eager calls between the replays."""
    c = Call([1400, 37], [1300, 2], 10, 2, 128, e4m3=e4m3, seed=61, max_new=1450, pad=200, bound=1800, width=120,
             k_gain=8.0, sm_scale=0.5)
    c.run()
    check(c)
    first = c.out.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        c.run()
    for _ in range(3):
        c.out.fill_(7.0)
        c.ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, first)
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(c.out, first)


def test_more_short_runs_than_tiles_of_32_rows():
    B, held, n, hq, hkv = MOST_TILES
    d = 64
    lens = [n + b % (held - n + 1) for b in range(B)]
    cache = Cache(lens, hkv, d, seed=71)
    shape = D().make_shape(B, hq, hkv, d, cache.width, held)
    q = queries(B * n, hq, d, 72)
    out = torch.full((B * n, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    off = torch.arange(0, B * n + 1, n, dtype=torch.int32, device="cuda")
    E().delta_extend_attn(shape, cache.on_gpu(D()), q.cuda(), out, off, n,
                          E().alloc_extend_workspace(shape, B * n, n))
    torch.cuda.synchronize()
    assert not bool(out.isnan().any())
    for b in (0, 1, 2, 255, 256, 8191, 8192, 16000, B - 1):
        for j in (0, 7, n - 1):
            t = range(lens[b] - n + j + 1)
            want, tol = attend(q[b * n + j], cache.tokens(0, b, t), cache.tokens(1, b, t), default_scale(d), P_ROUND)
            assert worst(out[b * n + j], want, tol) <= 1, (b, j)
