"""delta_tree_layout and delta_tree_attn against plain walks and float64: trees of every kind and size,
masks of any bits, ragged sequences, every group size, both cache types, tiles and splits of every kind."""
import pytest
import torch

from cache_cases import Cache, attend, default_scale, queries, worst
from draft_cases import mask_words, offsets_of, sees_of, tree
from gpu_helpers import D

pytestmark = pytest.mark.gpu

P_ROUND = 2.0 ** -8   # probabilities are rounded to bf16 before they meet the values


def T():
    from paper_2510_09883_amd import drafts
    return drafts


# ---- layout ------------------------------------------------------------------------------

def layout(lens, runs, words=None, pad=0, max_new=None, want=("positions", "masks"), offsets=True):
    """Positions and masks [rows, words] of runs of parents; rows that are not written hold -5."""
    rows = sum(map(len, runs)) + pad
    longest = max(map(len, runs))
    max_new = longest if max_new is None else max_new
    words = words or max(1, -(-max_new // 32))
    parents = torch.tensor([p for r in runs for p in r] + [3] * pad, dtype=torch.int32).cuda()
    pos = torch.full((rows,), -5, dtype=torch.int32, device="cuda")
    masks = torch.full((rows, words), -5, dtype=torch.int32, device="cuda")
    width = max(1, -(-max(lens) // 16))
    shape = D().make_shape(len(lens), 4, 1, 64, width, max(1, max(lens)))
    T().delta_tree_layout(shape, torch.tensor(lens, dtype=torch.int32).cuda(), parents,
                          pos if "positions" in want else None, masks if "masks" in want else None,
                          offsets_of([len(r) for r in runs]).cuda() if offsets else None, max_new)
    torch.cuda.synchronize()
    return pos.cpu(), masks.cpu()


def check_layout(lens, runs, words=None, pad=0, max_new=None, **kw):
    pos, masks = layout(lens, runs, words, pad, max_new, **kw)
    at = 0
    for s, run in zip(lens, runs):
        depths, sets = sees_of(run)
        n = len(run) if max_new is None else min(len(run), max_new)
        if n:
            assert pos[at:at + n].tolist() == [s - len(run) + x for x in depths[:n]]
            assert torch.equal(masks[at:at + n], mask_words(sets[:n], masks.shape[1]))
        assert bool((pos[at + n:at + len(run)] == -5).all() and (masks[at + n:at + len(run)] == -5).all())
        at += len(run)
    assert bool((pos[at:] == -5).all() and (masks[at:] == -5).all())


@pytest.mark.parametrize("kind", ["chain", "star", "pairs", "roots", "bush"])
def test_layout_of_trees(kind):
    sizes = [1, 0, 2, 31, 32, 33, 64, 65, 3, 127, 256, 257, 512]
    runs = [tree(n, kind, seed=n) for n in sizes]
    check_layout([n + 7 * i for i, n in enumerate(sizes)], runs, pad=2)
    check_layout([100, 5], [tree(9, kind), tree(4, kind)], words=5, max_new=9)


def test_layout_of_single_rows_and_many_sequences():
    check_layout([5, 1, 70], [[-1]] * 3, offsets=False)
    runs = [tree(b % 5, "bush", seed=b) for b in range(700)]
    check_layout([9 + b % 60 for b in range(700)], runs)


def test_layout_of_parents_that_name_no_row():
    """Itself, a later row, a row past the run, far negative: such a row continues nothing."""
    check_layout([40], [[-1, 1, 0, 7, 2, -9, 2 ** 31 - 1, -2 ** 31, 6]])


def test_layout_writes_no_more_than_it_is_asked_for():
    runs = [tree(40, "bush", 1), tree(7, "chain")]
    check_layout([50, 20], runs, max_new=33, words=2)       # places from max_new on are left
    pos, masks = layout([50, 20], runs, want=("positions",))
    assert bool((masks == -5).all()) and bool((pos != -5).all())
    pos, masks = layout([50, 20], runs, want=("masks",))
    assert bool((pos == -5).all()) and bool((masks[:, 0] != -5).all())


def test_layout_refusals():
    shape = D().make_shape(2, 4, 1, 64, 4, 64)
    p = torch.zeros(6, dtype=torch.int32, device="cuda")
    lens, off = p[:2].contiguous(), offsets_of([2, 4]).cuda()
    masks = torch.zeros((6, 1), dtype=torch.int32, device="cuda")
    err = D().DeltaError
    for error, match, args in [
            (ValueError, "^parents: expected", (lens, p.long(), p, masks, off, 4)),
            (ValueError, "^positions: expected", (lens, p, p[:5], masks, off, 4)),
            (ValueError, "^masks: expected", (lens, p, p, masks[:5], off, 4)),
            (ValueError, "^seq_lens: expected", (p, p, p, masks, off, 4)),
            (ValueError, "^row_offsets", (lens, p, p, masks, off[:2], 4)),
            (err, "invalid argument", (lens, p, None, None, off, 4)),
            (err, "invalid argument", (lens, p, p, masks, off, 7)),
            (err, "invalid argument", (lens, p, p, masks, None, 4)),
            (err, "invalid argument", (lens, p, p, masks[:, :0].contiguous(), off, 4))]:
        with pytest.raises(error, match=match):
            T().delta_tree_layout(shape, *args)
    many = torch.zeros(600, dtype=torch.int32, device="cuda")
    with pytest.raises(err, match="unsupported"):
        T().delta_tree_layout(shape, lens, many, many, None, offsets_of([0, 600]).cuda(), 513)


# ---- attention ---------------------------------------------------------------------------

class Call:
    """sets: for every run a list of sets of places that its rows see (default: those of `kind` trees)."""

    def __init__(self, lens, new, hq, hkv, d, e4m3=False, seed=0, pad=0, max_new=None, bound=None, width=None,
                 k_gain=1.0, sm_scale=0.0, kind="bush", sets=None, words=None, offsets=True):
        self.lens, self.new, self.hq = lens, new, hq
        self.cache = Cache(lens, hkv, d, e4m3=e4m3, seed=seed, width=width, k_gain=k_gain)
        self.rows = sum(new) + pad
        self.q = queries(self.rows, hq, d, seed + 1)
        self.scale = sm_scale or default_scale(d)
        self.kv = self.cache.on_gpu(D())
        self.shape = D().make_shape(len(lens), hq, hkv, d, self.cache.width, bound or max(max(lens), 1), sm_scale)
        self.max_new = max(new) if max_new is None else max_new
        self.sets = sets or [sees_of(tree(n, kind, seed + b))[1] for b, n in enumerate(new)]
        words = words or max(1, -(-self.max_new // 32))
        masks = mask_words([s for run in self.sets for s in run], words)
        self.masks = torch.cat([masks, torch.full((pad, words), -1, dtype=torch.int32)]).cuda()
        self.offsets = offsets_of(new).cuda() if offsets else None
        self.gpu = self.q.cuda()
        if pad:
            self.gpu[sum(new):] = float("nan")
        self.out = torch.full_like(self.gpu, 7.0)
        self.ws = T().alloc_tree_workspace(self.shape, self.rows, self.max_new)
        self.ws.fill_(0xFF)   # of any content

    def run(self):
        T().delta_tree_attn(self.shape, self.kv, self.gpu, self.out, self.masks, self.offsets, self.max_new, self.ws)

    def tokens(self, b, j):
        before = self.lens[b] - self.new[b]
        seen = sorted(i for i in self.sets[b][j] if i < self.new[b] and before + i >= 0)
        return list(range(max(0, before))) + [before + i for i in seen]

    def check(self, some=None):
        """Every row, or the first, the last and `some` in between of every run."""
        torch.cuda.synchronize()
        out = self.out.cpu()
        row = 0
        for b, n in enumerate(self.new):
            picks = range(n)
            if some is not None and n > some + 2:
                g = torch.Generator().manual_seed(b)
                picks = sorted({0, n - 1, *torch.randint(0, n, (some,), generator=g).tolist()})
            for j in picks:
                t = self.tokens(b, j)
                want, tol = attend(self.q[row + j], self.cache.tokens(0, b, t), self.cache.tokens(1, b, t),
                                   self.scale, P_ROUND)
                assert worst(out[row + j], want, tol) <= 1, f"row {j} of run {b} ({n} of {self.lens[b]} tokens)"
            row += n
        assert bool((out[row:] == 7.0).all()), "rows behind the last run were written"


@pytest.mark.parametrize("G,hkv,d", [(1, 2, 128), (2, 1, 64), (3, 2, 128), (4, 8, 128), (5, 2, 64), (6, 2, 128),
                                     (7, 4, 128), (8, 2, 64)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_small_trees(G, hkv, d, e4m3):
    lens = [0, 1, 4, 15, 16, 17, 100, 257, 600]
    c = Call(lens, [0, 1, 4, 3, 2, 1, 4, 0, 3], G * hkv, hkv, d, e4m3=e4m3, seed=G, pad=2)
    c.run()
    c.check()


@pytest.mark.parametrize("G,hkv,d", [(1, 1, 64), (2, 2, 128), (4, 2, 128), (5, 1, 128), (7, 1, 64), (8, 1, 128)])
@pytest.mark.parametrize("kind", ["bush", "pairs"])
@pytest.mark.parametrize("e4m3", [False, True])
def test_trees_of_every_size(G, hkv, d, kind, e4m3):
    """Around the tiles' and the mask words' edges, behind prefixes that end anywhere in a block."""
    lens = [150, 64, 1, 300, 33, 513, 40, 130, 95]
    new = [16, 63, 1, 32, 0, 130, 33, 65, 31]
    c = Call(lens, new, G * hkv, hkv, d, e4m3=e4m3, seed=20 + G, pad=5, kind=kind)
    c.run()
    c.check(some=16)


@pytest.mark.parametrize("nodes", [8, 9, 16, 17, 32, 33, 64, 65, 100])
@pytest.mark.parametrize("e4m3", [False, True])
def test_trees_of_one_size(nodes, e4m3):
    """All runs alike, so that every kernel that the size picks is met."""
    for G in (4, 7):
        c = Call([nodes, 400 + nodes, 1000, 37 + nodes], [nodes] * 4, 2 * G, 2, 128, e4m3=e4m3, seed=nodes)
        c.run()
        c.check(some=12)


@pytest.mark.parametrize("kind", ["chain", "star", "roots"])
def test_the_longest_trees(kind):
    c = Call([512, 900], [512, 300], 4, 2, 64, seed=5, kind=kind)
    c.run()
    c.check(some=30)


def test_a_chain_is_a_causal_run():
    from paper_2510_09883_amd import extend as E
    c = Call([300, 77, 20], [40, 9, 20], 8, 2, 128, seed=6, kind="chain")
    c.run()
    c.check()
    out = torch.zeros_like(c.out)
    E.delta_extend_attn(c.shape, c.kv, c.gpu, out, c.offsets, 40, E.alloc_extend_workspace(c.shape, c.rows, 40))
    torch.cuda.synchronize()
    # both within their own bounds of the same result: two bf16 steps and the rounded probabilities
    assert float((out.float() - c.out.float()).abs().max()) <= 3 * 2.0 ** -8 * 4


@pytest.mark.parametrize("new", [1, 3, 20, 40, 90])
@pytest.mark.parametrize("e4m3", [False, True])
def test_few_rows_of_a_long_cache_are_split(new, e4m3):
    """One sequence: the cache's length is cut into pieces and joined; a bound far above the length leaves
    pieces without keys."""
    for length, bound in ((9000, 9000), (700, 16000), (new, 16000)):
        c = Call([length], [new], 4, 1, 128, e4m3=e4m3, seed=new, bound=bound, width=1000)
        c.run()
        c.check(some=12)


def test_masks_of_any_bits():
    """Rows that do not see themselves, that see later rows, all, or none; bits past the run are ignored."""
    g = torch.Generator().manual_seed(9)
    for lens, new in (([70, 33, 40], [40, 33, 7]), ([300, 20], [100, 20])):
        sets = []
        for n in new:
            run = [frozenset(torch.nonzero(torch.rand((n + 9,), generator=g) < 0.4).flatten().tolist()) for _ in range(n)]
            run[0], run[n // 2], run[n - 1] = frozenset(), frozenset(range(n + 9)), frozenset({0})
            sets.append(run)
        for e4m3 in (False, True):
            c = Call(lens, new, 8, 2, 128, e4m3=e4m3, seed=len(lens), sets=sets, words=4)
            c.run()
            c.check()


def test_rows_that_see_nothing_are_zeros():
    """Whole sequences of drafts with empty masks, and lengths below the run's."""
    c = Call([40, 7, 3], [40, 7, 9], 8, 2, 64, seed=10, sets=[[frozenset()] * 40, [frozenset()] * 7,
                                                           [frozenset({j}) for j in range(9)]])
    c.run()
    c.check()
    assert not c.out[:47].any() and not c.out[47:53].any() and bool(c.out[53:].any())
    c = Call([0, 90], [5, 90], 8, 2, 128, seed=11, sets=[[frozenset({0, 1})] * 5, [frozenset()] * 45 + [frozenset({3})] * 45])
    c.run()
    c.check(some=20)


def test_single_rows_without_offsets():
    lens = [1, 31, 500, 1024]
    c = Call(lens, [1] * 4, 8, 2, 128, seed=43, offsets=False)
    c.run()
    c.check()
    full = torch.empty_like(c.out)
    D().delta_full_attn(c.shape, c.kv, c.gpu, full, D().alloc_workspace(c.shape))
    torch.cuda.synchronize()
    assert float((full.float() - c.out.float()).abs().max()) <= 3 * 2.0 ** -8 * 4


@pytest.mark.parametrize("batch", [65, 257, 700])
def test_many_sequences(batch):
    lens = [(17 * b) % 50 + 4 for b in range(batch)]
    new = [max(0, (b * 5) % 5 - 1) if b % 3 else 0 for b in range(batch)]
    lens[-1], new[-1] = 90, 80
    c = Call(lens, new, 4, 2, 64, seed=batch, pad=3)
    c.run()
    c.check(some=4)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("held,new,at", [(60, 6, 57), (300, 8, 294), (500, 120, 430), (130, 130, 0), (700, 400, 301),
                                         (260, 70, 200)])
def test_values_of_tokens_that_a_row_does_not_see_do_not_reach_it(held, new, at, e4m3):
    """Token `at` has an infinite (e4m3: NaN) value element and token at + 2 a key of NaN."""
    c = Call([held, 20], [new, 3], 8, 2, 128, e4m3=e4m3, seed=held)
    k, v = c.kv._tensors[:2]
    place = lambda t: (int(c.cache.table[0, t // 16]), slice(None), t % 16)   # noqa: E731
    raw = v.view(torch.uint8 if e4m3 else torch.int16)
    raw[place(at)][:, 5] = 0x7F if e4m3 else 0x7F80
    if at + 2 < held:
        k.view(raw.dtype)[place(at + 2)] = 0x7F if e4m3 else 0x7FC0
    c.run()
    torch.cuda.synchronize()
    out = c.out.cpu()
    for j in range(0, new, max(1, new // 60)):
        t = c.tokens(0, j)
        if at + 2 in t:
            assert bool(out[j].isnan().all()), j
            continue
        want, tol = attend(c.q[j], c.cache.tokens(0, 0, t), c.cache.tokens(1, 0, t), c.scale, P_ROUND)
        got = out[j].clone()
        if at in t:
            assert not bool(got[:, 5].isfinite().any()), j
            got[:, 5] = want[:, 5].to(got.dtype)
        assert worst(got, want, tol) <= 1, j
    t = c.tokens(1, 0)
    want, tol = attend(c.q[new], c.cache.tokens(0, 1, t), c.cache.tokens(1, 1, t), c.scale, P_ROUND)
    assert worst(out[new], want, tol) <= 1


def test_a_query_of_nan_spoils_its_own_outputs_only():
    for new in (3, 20, 90):
        c = Call([120], [new], 8, 2, 128, seed=52)
        c.gpu[1, 2] = float("nan")
        c.run()
        torch.cuda.synchronize()
        assert bool(c.out[1, 2].isnan().all())
        c.out[1, 2] = 0
        assert not bool(c.out.isnan().any())


def test_sharp_scores_and_a_larger_bound_of_the_runs():
    for new in ([2, 5], [20, 30], [90, 200]):
        c = Call([90, 300], new, 8, 2, 128, seed=46, max_new=max(new) + 2, pad=200, k_gain=8.0, sm_scale=0.5)
        c.run()
        c.check(some=30)


def test_equal_calls_give_equal_bits_and_graph_replays():
    for new in ([3, 5, 8], [20, 33, 64]):
        c = Call([2000, 77, 900], new, 16, 2, 128, e4m3=True, seed=49)
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

    def call(error, match, shape=c.shape, q=c.gpu, out=c.out, masks=c.masks, off=c.offsets, max_new=3, ws=c.ws):
        with pytest.raises(error, match=match):
            T().delta_tree_attn(shape, c.kv, q, out, masks, off, max_new, ws)
    call(ValueError, "^q: expected shape", q=c.gpu[:, :4].contiguous())
    call(ValueError, "^out: expected shape", out=c.out[:3])
    call(ValueError, "^masks: expected shape", masks=c.masks[:4])
    call(ValueError, "^masks: expected torch.int32", masks=c.masks.long())
    call(ValueError, "^row_offsets", off=c.offsets.long())
    call(err, "invalid argument", masks=c.masks[:, :0].contiguous())
    call(err, "invalid argument", off=None)
    call(err, "invalid argument", max_new=-1)
    call(err, "invalid argument", max_new=6)
    call(err, "workspace too small", ws=c.ws[:8])
    off_by_8 = torch.zeros(c.ws.numel() + 64, dtype=torch.uint8, device="cuda")[8:]
    call(err, "invalid argument", ws=off_by_8)
    torch.cuda.synchronize()
    assert bool((c.out == 7.0).all())
