"""delta_extend_attn against float64: ragged runs from no token to long ones, every group size, both
cache types, tiles and splits of every kind, and rows that see nothing."""
import pytest
import torch

from cache_cases import Cache, attend, default_scale, queries, worst
from gpu_helpers import D

pytestmark = pytest.mark.gpu

P_ROUND = 2.0 ** -8   # probabilities are rounded to bf16 before they meet the values


def E():
    from paper_2510_09883_amd import extend
    return extend


class Call:
    def __init__(self, lens, new, hq, hkv, d, e4m3=False, seed=0, pad=0, max_new=None, bound=None, width=None,
                 k_gain=1.0, sm_scale=0.0, offsets=True):
        self.lens, self.new, self.hq = lens, new, hq
        self.cache = Cache(lens, hkv, d, e4m3=e4m3, seed=seed, width=width, k_gain=k_gain)
        self.rows = sum(new) + pad
        self.q = queries(self.rows, hq, d, seed + 1)
        self.scale = sm_scale or default_scale(d)
        self.kv = self.cache.on_gpu(D())
        self.shape = D().make_shape(len(lens), hq, hkv, d, self.cache.width, bound or max(max(lens), 1), sm_scale)
        self.max_new = max(new) if max_new is None else max_new
        self.offsets = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32).cuda() if offsets else None
        self.gpu = self.q.cuda()
        if pad:
            self.gpu[sum(new):] = float("nan")
        self.out = torch.full_like(self.gpu, 7.0)
        self.ws = E().alloc_extend_workspace(self.shape, self.rows, self.max_new)
        self.ws.fill_(0xFF)   # of any content

    def run(self):
        E().delta_extend_attn(self.shape, self.kv, self.gpu, self.out, self.offsets, self.max_new, self.ws)

    def check(self, some=None):
        """Every row, or the first, the last and `some` in between of every run."""
        torch.cuda.synchronize()
        out = self.out.cpu()
        row = 0
        for b, (s, n) in enumerate(zip(self.lens, self.new)):
            picks = range(n)
            if some is not None and n > some + 2:
                g = torch.Generator().manual_seed(b)
                picks = sorted({0, n - 1, *torch.randint(0, n, (some,), generator=g).tolist()})
            for j in picks:
                t = range(max(0, s - n + j + 1))
                want, tol = attend(self.q[row + j], self.cache.tokens(0, b, t), self.cache.tokens(1, b, t),
                                   self.scale, P_ROUND)
                assert worst(out[row + j], want, tol) <= 1, f"row {j} of run {b} ({n} of {s} tokens)"
            row += n
        assert bool((out[row:] == 7.0).all()), "rows behind the last run were written"


@pytest.mark.parametrize("G,hkv,d", [(1, 2, 128), (2, 1, 64), (3, 2, 128), (4, 8, 128), (5, 2, 64), (6, 2, 128),
                                     (7, 4, 128), (8, 2, 64)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_short_runs(G, hkv, d, e4m3):
    """Runs that fit a small tile, none to four tokens, at ragged lengths."""
    lens = [0, 1, 4, 15, 16, 17, 100, 257, 600]
    c = Call(lens, [0, 1, 4, 3, 2, 1, 4, 0, 3], G * hkv, hkv, d, e4m3=e4m3, seed=G, pad=2)
    c.run()
    c.check()


@pytest.mark.parametrize("G,hkv,d", [(1, 1, 64), (2, 2, 128), (4, 2, 128), (5, 1, 128), (7, 1, 64), (8, 1, 128)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_prompts_and_chunks(G, hkv, d, e4m3):
    """Whole prompts and chunks behind a prefix, beside single tokens and empty runs."""
    lens = [150, 64, 1, 300, 33, 513, 40]
    new = [150, 63, 1, 70, 0, 130, 1]
    c = Call(lens, new, G * hkv, hkv, d, e4m3=e4m3, seed=20 + G, pad=5)
    c.run()
    c.check(some=24)


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_long_prompt(e4m3):
    c = Call([2500], [2500], 8, 2, 128, e4m3=e4m3, seed=31)
    c.run()
    c.check(some=60)


@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("e4m3", [False, True])
def test_few_rows_of_a_long_cache_are_split(new, e4m3):
    """One sequence: the cache's length is cut into pieces and joined; a bound far above the length
    leaves pieces without keys."""
    for length, bound in ((9000, 9000), (700, 16000), (new, 16000)):
        c = Call([length], [new], 4, 1, 128, e4m3=e4m3, seed=new, bound=bound, width=1000)
        c.run()
        c.check()


def test_many_sequences():
    """More sequences than a wave has lanes, with empty runs between them."""
    lens = [(29 * b) % 140 + 3 for b in range(200)]
    new = [(b * 7) % 4 for b in range(200)]
    c = Call(lens, new, 6, 2, 64, seed=41)
    c.run()
    c.check()
    c = Call(lens, [0] * 199 + [120], 6, 2, 64, seed=42)
    c.lens[199] = lens[199] = max(lens[199], 120)
    c = Call(lens, [0] * 199 + [120], 6, 2, 64, seed=42, pad=1)
    c.run()
    c.check()


@pytest.mark.parametrize("batch", [65, 256, 257, 700])
def test_batches_around_what_a_lane_holds(batch):
    """Runs of every length around the tile, empty ones among them, and one long one at the end."""
    lens = [(17 * b) % 50 + 4 for b in range(batch)]
    new = [(b * 5) % 5 - 1 if b % 3 else 0 for b in range(batch)]
    new = [max(0, n) for n in new]
    lens[-1], new[-1] = 90, 80
    c = Call(lens, new, 4, 2, 64, seed=batch, pad=3)
    c.run()
    c.check(some=4)


def test_a_query_of_nan_spoils_its_own_outputs_only():
    for new in (3, 90):
        c = Call([120], [new], 8, 2, 128, seed=52)
        c.gpu[1, 2] = float("nan")
        c.run()
        torch.cuda.synchronize()
        assert bool(c.out[1, 2].isnan().all())
        c.out[1, 2] = 0
        assert not bool(c.out.isnan().any())


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("held,new,at", [(60, 6, 57), (300, 8, 294), (500, 120, 430), (130, 130, 0), (700, 400, 301),
                                         (260, 70, 200)])
def test_values_of_tokens_that_a_row_does_not_see_do_not_reach_it(held, new, at, e4m3):
    """Token `at` has an infinite (e4m3: NaN) value element and the token after it a key of NaN: rows
    before them are as if both were not there, rows that see the value have it in that element alone, rows
    that see the key are NaN."""
    c = Call([held, 20], [new, 3], 8, 2, 128, e4m3=e4m3, seed=held)
    k, v = c.kv._tensors[:2]
    place = lambda t: (int(c.cache.table[0, t // 16]), slice(None), t % 16)   # noqa: E731
    raw = v.view(torch.uint8 if e4m3 else torch.int16)
    raw[place(at)][:, 5] = 0x7F if e4m3 else 0x7F80
    if at + 1 < held:
        k.view(raw.dtype)[place(at + 1)] = 0x7F if e4m3 else 0x7FC0
    c.run()
    torch.cuda.synchronize()
    out = c.out.cpu()
    for j in sorted({*range(0, new, max(1, new // 40)), *(x for x in (at - held + new - 1, at - held + new,
                                                                     at - held + new + 1) if 0 <= x < new)}):
        last = held - new + j
        if last > at:
            assert bool(out[j].isnan().all()), j     # it sees the key of NaN
            continue
        keys = c.cache.tokens(0, 0, range(last + 1))
        values = c.cache.tokens(1, 0, range(last + 1))
        want, tol = attend(c.q[j], keys, values, c.scale, P_ROUND)
        got = out[j].clone()
        if last == at:
            assert not bool(got[:, 5].isfinite().any()), j
            got[:, 5] = want[:, 5].to(got.dtype)
        assert worst(got, want, tol) <= 1, j
    want, tol = attend(c.q[new], c.cache.tokens(0, 1, range(18)), c.cache.tokens(1, 1, range(18)), c.scale, P_ROUND)
    assert worst(out[new], want, tol) <= 1


def test_single_tokens_without_offsets_match_the_decode_layer():
    lens = [1, 31, 500, 1024]
    c = Call(lens, [1] * 4, 8, 2, 128, seed=43, offsets=False)
    c.run()
    c.check()
    full = torch.empty_like(c.out)
    D().delta_full_attn(c.shape, c.kv, c.gpu, full, D().alloc_workspace(c.shape))
    torch.cuda.synchronize()
    # both within their own bounds of the same result: two bf16 steps and the rounded probabilities
    assert float((full.float() - c.out.float()).abs().max()) <= 3 * 2.0 ** -8 * 4


def test_rows_that_see_nothing_are_zeros():
    """A length below the run's: the run's first rows are tokens before the sequence's first."""
    for new in (6, 200):
        c = Call([4, 40], [new, 10], 8, 2, 128, seed=44)
        c.run()
        c.check(some=40)
        assert not c.out[:new - 4].any()
    c = Call([0, 9], [3, 2], 8, 2, 64, seed=45)
    c.run()
    c.check()
    assert not c.out[:3].any()


def test_a_larger_bound_of_the_runs_and_sharp_scores():
    c = Call([90, 300], [2, 5], 8, 2, 128, seed=46, max_new=7, pad=200, k_gain=8.0, sm_scale=0.5)
    c.run()
    c.check()
    c = Call([90, 300], [90, 200], 8, 2, 128, seed=47, max_new=250, k_gain=8.0, sm_scale=0.5)
    c.run()
    c.check(some=40)


def test_large_scores_keep_their_order():
    """Scores of 1e12: the largest alone counts, equal ones share."""
    for new in (2, 70):
        c = Call([200], [new], 4, 1, 128, seed=48)
        k, v = c.kv._tensors[:2]
        x = torch.zeros_like(k.float())
        for t, val in ((3, 1e6), (60, 1e6), (100, 9.9e5)):
            x[c.cache.table[0, t // 16], 0, t % 16, 0] = val
        k.copy_(x.to(torch.bfloat16))
        c.gpu.zero_()
        c.gpu[..., 0] = 1e7
        c.run()
        torch.cuda.synchronize()
        vals = torch.stack([v[c.cache.table[0, t // 16], 0, t % 16].float() for t in (3, 60)])
        want = vals.mean(0).to(torch.bfloat16)
        assert torch.equal(c.out, want.expand_as(c.out))


def test_equal_calls_give_equal_bits_and_graph_replays():
    lens = [2000, 77, 900]
    c = Call(lens, [3, 5, 8], 16, 2, 128, e4m3=True, seed=49)
    c.run()
    torch.cuda.synchronize()
    first = c.out.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        c.run()
    for _ in range(4):
        c.out.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, first)
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(c.out, first)


def test_no_rows_and_refusals():
    c = Call([5, 9], [0, 0], 8, 2, 64, seed=50)
    c.run()
    c.check()
    c = Call([20, 30], [2, 3], 8, 2, 64, seed=51)
    err = D().DeltaError

    def call(error, match, shape=c.shape, q=c.gpu, out=c.out, off=c.offsets, max_new=3, ws=c.ws):
        with pytest.raises(error, match=match):
            E().delta_extend_attn(shape, c.kv, q, out, off, max_new, ws)
    call(ValueError, "^q: expected shape", q=c.gpu[:, :4].contiguous())
    call(ValueError, "^out: expected shape", out=c.out[:3])
    call(ValueError, "^out: expected torch.bfloat16", out=c.out.float())
    call(ValueError, "^q: must be contiguous", q=torch.empty((5, 8, 128), dtype=torch.bfloat16, device="cuda")[..., ::2])
    call(ValueError, "^row_offsets", off=c.offsets.long())
    call(err, "invalid argument", off=None)
    call(err, "invalid argument", max_new=-1)
    call(err, "invalid argument", max_new=6)
    call(err, "workspace too small", ws=c.ws[:8])
    off_by_8 = torch.zeros(c.ws.numel() + 64, dtype=torch.uint8, device="cuda")[8:]
    call(err, "invalid argument", ws=off_by_8)
    torch.cuda.synchronize()
    assert bool((c.out == 7.0).all())
