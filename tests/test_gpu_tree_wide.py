"""delta_tree_attn's tiles of 256 rows against float64, every row: both head sizes and cache types, tiles of up to
128 rows and more, pieces, equal shares and calls that are not shared, infinite and NaN values, masks of any bits,
rows that see nothing, long page lists, pages past 32 bits, and captured calls."""
import pytest
import torch

import wide_tree_cases as C
from cache_cases import PAGE, default_scale, worst
from draft_cases import mask_words, offsets_of, sees_of, tree
from gpu_helpers import D
from test_gpu_tree_attn import Call, T

pytestmark = pytest.mark.gpu

BOTH = [(64, False), (64, True), (128, False), (128, True)]


def call(case, d, e4m3, **kw):
    lens, new, hq, hkv, bound = case
    kw.setdefault("width", -(-(bound or max(lens)) // PAGE))
    return Call(list(lens), list(new), hq, hkv, d, e4m3=e4m3, bound=bound, **kw)


def check(c):
    torch.cuda.synchronize()
    out = c.out.cpu()
    want, tol = C.attend_runs(c)
    n = want.shape[0]
    row = 0
    for b, k in enumerate(c.new):
        if k:
            off = worst(out[row:row + k], want[row:row + k], tol[row:row + k])
            assert off <= 1, f"run {b} ({k} of {c.lens[b]} tokens): {off}"
        row += k
    assert bool((out[n:] == 7.0).all()), "rows behind the last run were written"


@pytest.mark.parametrize("d,e4m3", BOTH)
@pytest.mark.parametrize("case", range(len(C.WIDE)))
def test_tiles_of_256_rows(case, d, e4m3):
    c = call(C.WIDE[case], d, e4m3, seed=100 + case, pad=3, kind=("bush", "pairs", "chain")[case % 3])
    c.run()
    check(c)


@pytest.mark.parametrize("d,e4m3", BOTH)
@pytest.mark.parametrize("case", range(30))
def test_drawn_calls(case, d, e4m3):
    c = call(C.drawn(30)[case], d, e4m3, seed=case, pad=3)
    c.run()
    check(c)


@pytest.mark.parametrize("d,e4m3", BOTH)
@pytest.mark.parametrize("case", C.HIDDEN)
def test_values_of_tokens_that_a_row_does_not_see(case, d, e4m3):
    """Token `at` has an infinite (e4m3: NaN) value element and token at + 2 a key of NaN."""
    at = case[1]
    c = call(C.hidden_call(case), d, e4m3, seed=at)
    held, new = c.lens[0], c.new[0]
    k, v = c.kv._tensors[:2]
    place = lambda t: (int(c.cache.table[0, t // PAGE]), slice(None), t % PAGE)   # noqa: E731
    raw = v.view(torch.uint8 if e4m3 else torch.int16)
    raw[place(at)][:, 5] = 0x7F if e4m3 else 0x7F80
    if at + 2 < held:
        k.view(raw.dtype)[place(at + 2)] = 0x7F if e4m3 else 0x7FC0
    c.run()
    torch.cuda.synchronize()
    out = c.out.cpu()
    want, tol = C.attend_runs(c)   # (from what the cache held before)
    for j in range(new):
        t = c.tokens(0, j)
        if at + 2 in t:
            assert bool(out[j].isnan().all()), j
            continue
        got = out[j].clone()
        if at in t:
            assert not bool(got[:, 5].isfinite().any()), j
            got[:, 5] = want[j, :, 5].to(got.dtype)
        assert worst(got, want[j], tol[j]) <= 1, j
    assert worst(out[new:], want[new:], tol[new:]) <= 1


@pytest.mark.parametrize("d,e4m3", BOTH)
def test_masks_of_any_bits(d, e4m3):
    """Rows that do not see themselves, that see later rows, all, or none; bits past the run are ignored."""
    g = torch.Generator().manual_seed(9)
    sets = []
    for n in C.BITS[1]:
        run = [frozenset(torch.nonzero(torch.rand((n + 9,), generator=g) < 0.4).flatten().tolist()) for _ in range(n)]
        run[0], run[n // 2], run[n - 1] = frozenset(), frozenset(range(n + 9)), frozenset({0})
        sets.append(run)
    c = call(C.BITS, d, e4m3, seed=7, sets=sets, words=5)
    c.run()
    check(c)


@pytest.mark.parametrize("d,e4m3", BOTH)
def test_rows_that_see_nothing_are_zeros(d, e4m3):
    """Empty masks where the run is the whole sequence, or the sequence is empty."""
    new = C.NOTHING[1]
    sets = [[frozenset({j}) for j in range(100)], [frozenset()] * 45 + [frozenset({3})] * 45, [frozenset()] * 64,
            [frozenset({0, 1})] * 5]
    c = call(C.NOTHING, d, e4m3, seed=8, sets=sets)
    c.run()
    check(c)
    first = new[0]
    assert not c.out[first:first + 45].any() and bool(c.out[first + 45:first + 90].any())
    assert not c.out[first + 90:].any()


@pytest.mark.parametrize("d,e4m3", BOTH)
def test_sharp_scores_and_a_larger_bound_of_the_runs(d, e4m3):
    c = call(C.SHARP, d, e4m3, seed=46, max_new=max(C.SHARP[1]) + 2, pad=200, k_gain=8.0, sm_scale=0.5)
    c.run()
    check(c)


@pytest.mark.parametrize("d,e4m3", BOTH)
@pytest.mark.parametrize("case", range(len(C.REPLAYS)))
def test_equal_calls_give_equal_bits_and_graph_replays(case, d, e4m3):
    c = call(C.REPLAYS[case], d, e4m3, seed=49)
    c.run()
    check(c)
    first = c.out.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        c.run()
    for _ in range(4):
        c.out.fill_(3.0)
        c.ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, first)
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(c.out, first)


@pytest.mark.parametrize("d,e4m3", BOTH)
def test_more_pages_than_are_looked_up_at_a_time(d, e4m3):
    """Sequences of more than 1024 pages, in a call of more sequences than are shared out."""
    c = call(C.pages_call(), d, e4m3, seed=50)
    c.run()
    check(c)


@pytest.mark.parametrize("batch", [65, 257, 700])
@pytest.mark.parametrize("e4m3", [False, True])
def test_many_sequences_with_rows(batch, e4m3):
    """Most of the sequences have a run of one to four rows: more than a wave counts at a time, and more than
    are shared out; in tiles of 32 rows, and beside a long run in tiles of 256."""
    for longest, d in ((4, 128), (80, 64)):
        new = [b % 5 for b in range(batch)]
        lens = [(17 * b) % 50 + 4 for b in range(batch)]
        lens[batch // 2], new[batch // 2] = 900, longest
        c = Call(lens, new, 8, 2, d, e4m3=e4m3, seed=batch, pad=3)
        c.run()
        check(c)


@pytest.mark.parametrize("e4m3", [False, True])
def test_pages_past_32_bits(e4m3):
    """More than 2^32 elements in a cache, pages at both ends."""
    (n, m), hq, hkv, bound = C.FAR
    d, pages = 128, 262144 + 40     # 2^32 elements are 262144 pages
    kind = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    k, v = (torch.zeros((pages, hkv, PAGE, d), dtype=torch.uint8 if e4m3 else torch.int16, device="cuda").view(kind)
            for _ in range(2))
    table = torch.zeros((1, bound // PAGE), dtype=torch.int32)
    table[0, :5] = torch.tensor([pages - 1, 7, 262144, pages - 3, 131072])
    g = torch.Generator().manual_seed(3)
    t = torch.arange(n)
    held = []
    for x in (k, v):
        rows = torch.randn((n, hkv, d), generator=g).to(kind)
        x.view(torch.uint8 if e4m3 else torch.int16)[table[0, t // PAGE].long().cuda(), :, (t % PAGE).cuda()] = \
            rows.view(torch.uint8 if e4m3 else torch.int16).cuda()
        held.append(rows.double())

    class Small:   # (what C.attend_runs looks at)
        lens, new, scale = [n], [m], default_scale(d)
        q = torch.randn((m, hq, d), generator=g).to(torch.bfloat16)
        sets = [sees_of(tree(m, "bush", 4))[1]]
        tokens = Call.tokens
    c = Small()
    c.hq, c.cache = hq, type("Heads", (), {"hkv": hkv})
    shape = D().make_shape(1, hq, hkv, d, bound // PAGE, bound)
    kv = D().make_kv(k, v, table.cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"))
    out = torch.zeros((m, hq, d), dtype=torch.bfloat16, device="cuda")
    T().delta_tree_attn(shape, kv, c.q.cuda(), out, mask_words(c.sets[0], 2).cuda(), offsets_of([m]).cuda(), m,
                        T().alloc_tree_workspace(shape, m, m))
    torch.cuda.synchronize()
    want, tol = C.attend_runs(c, lambda b: held[0], lambda b: held[1])
    assert worst(out, want, tol) <= 1
