"""Rounds of drafted tokens as a server runs them: trees are laid out, normed, rotated and appended, attended in
layers of both cache types, verified, and the accepted rows are kept; eagerly and replayed from a graph.  The
debug build's checks of the same calls, and caches and probabilities whose offsets pass 32 bits."""
import ctypes
import os

import pytest
import torch

from cache_cases import PAGE, attend, default_scale, worst
from draft_cases import mask_words, offsets_of, sees_of, tree, verified
from gpu_helpers import D
from test_gpu_norm_append import normed, turned
from test_gpu_rope_append import frequencies

pytestmark = pytest.mark.gpu

HQ, HKV, HD, VOCAB = 14, 2, 128, 700
P_ROUND = 2.0 ** -8


def T():
    from paper_2510_09883_amd import drafts
    return drafts


class Server:
    """Two layers, bf16 and e4m3, over one page table; a round has the same runs every time."""

    def __init__(self, new=(9, 1, 20), capacity=320, seed=1):
        self.new, self.B, self.width, self.rows = list(new), len(new), capacity // PAGE, sum(new) + 2
        g = torch.Generator().manual_seed(seed)
        self.g = g
        n = self.B * self.width
        self.table = torch.randperm(n, generator=g).int().view(self.B, self.width)
        table = self.table.cuda()
        self.lens = torch.zeros((self.B,), dtype=torch.int32, device="cuda")
        self.kinds = [torch.bfloat16, torch.float8_e4m3fn]
        self.scales = [None, [(0.02 + 0.05 * torch.rand((HKV,), generator=g)).cuda() for _ in range(2)]]
        self.caches = [[torch.full((n, HKV, PAGE, HD), float("nan")).to(kind).cuda() for _ in range(2)] for kind in self.kinds]
        self.kvs = [D().make_kv(*c, table, self.lens, *(s or [None, None])) for c, s in zip(self.caches, self.scales)]
        self.shape = D().make_shape(self.B, HQ, HKV, HD, self.width, capacity)
        self.weights = [(1 + 0.2 * torch.randn((HD,), generator=g)).to(torch.bfloat16) for _ in range(2)]
        self.w_gpu = [w.cuda() for w in self.weights]
        self.inv_freq = frequencies(HD, 1e6)
        self.f_gpu = self.inv_freq.cuda()
        self.offsets = offsets_of(self.new).cuda()
        self.runs = torch.tensor(self.new, dtype=torch.int32).cuda()
        self.max_new = max(self.new)
        words = -(-self.max_new // 32)
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")   # noqa: E731
        bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")   # noqa: E731
        self.parents, self.tokens, self.positions, self.masks = i32(self.rows), i32(self.rows), i32(self.rows), i32(self.rows, words)
        self.path, self.n_path, self.next = i32(self.B, self.max_new), i32(self.B), i32(self.B)
        self.qkv, self.q, self.out = [bf(self.rows, HQ + 2 * HKV, HD) for _ in range(2)], [bf(self.rows, HQ, HD) for _ in range(2)], \
            [bf(self.rows, HQ, HD) for _ in range(2)]
        self.target, self.draft = (torch.zeros((self.rows, VOCAB), device="cuda") for _ in range(2))
        self.uniform = torch.zeros((self.rows,), device="cuda")
        self.ws = T().alloc_tree_workspace(self.shape, self.rows, self.max_new)
        self.verify_ws = T().alloc_verify_workspace(self.B, VOCAB)
        self.stack = T().CacheStack(self.shape, self.kvs)

    def draw(self, seed):
        """A round's inputs, on the host and copied to where the calls read them."""
        g = torch.Generator().manual_seed(seed)
        x = dict(parents=[tree(n, "bush", seed + b) for b, n in enumerate(self.new)],
                 qkv=[torch.randn((self.rows, HQ + 2 * HKV, HD), generator=g).to(torch.bfloat16) for _ in range(2)])
        logits = 2.0 * torch.randn((self.rows, VOCAB), generator=g)
        x["target"] = torch.softmax(logits, -1)
        x["draft"] = torch.softmax(logits + 0.4 * torch.randn((self.rows, VOCAB), generator=g), -1)
        x["uniform"] = torch.rand((self.rows,), generator=g)
        x["tokens"], at = [0] * self.rows, 0
        for run in x["parents"]:
            for j, p in enumerate(run):
                x["tokens"][at + j] = int(torch.multinomial(x["draft"][at + max(p, 0)], 1, generator=g))
            at += len(run)
        flat = [p for run in x["parents"] for p in run] + [5, 5]
        for name, value in (("parents", torch.tensor(flat)), ("tokens", torch.tensor(x["tokens"])), ("target", x["target"]),
                            ("draft", x["draft"]), ("uniform", x["uniform"])):
            getattr(self, name).copy_(value)
        for dst, src in zip(self.qkv, x["qkv"]):
            dst.copy_(src)
        torch.cuda.synchronize()
        return x

    def round(self):
        """All calls of a round; the lengths grow by the runs, then shrink to what was accepted."""
        t = T()
        self.lens.add_(self.runs)
        t.delta_tree_layout(self.shape, self.lens, self.parents, self.positions, self.masks, self.offsets, self.max_new)
        for kv, qkv, q, out in zip(self.kvs, self.qkv, self.q, self.out):
            t.delta_norm_rope_append(self.shape, kv, qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], q, *self.w_gpu, 1e-6,
                                     self.f_gpu, row_offsets=self.offsets, positions=self.positions)
            t.delta_tree_attn(self.shape, kv, q, out, self.masks, self.offsets, self.max_new, self.ws)
        t.delta_verify_drafts(self.target, self.draft, self.tokens, self.parents, self.uniform, self.offsets, self.path,
                              self.n_path, self.next, self.verify_ws)
        t.delta_cache_compact(self.stack, self.rows, self.offsets, self.path, self.n_path, self.lens)

    def held(self, layer, which, b, n):
        """float64 [n, hkv, d] of what a cache holds for sequence b's first n tokens."""
        t = torch.arange(n)
        x = self.caches[layer][which].cpu().double()[self.table[b, t // PAGE].long(), :, t % PAGE]
        return x if self.scales[layer] is None else x * self.scales[layer][which].cpu().double()[:, None]

    def state(self):
        return [self.lens, self.positions, self.masks, self.path, self.n_path, self.next,
                *[o.view(torch.int16) for o in self.out], *[c.view(torch.uint8) for layer in self.caches for c in layer]]


def check_rounds(srv, n_rounds):
    kept = [[] for _ in range(srv.B)]   # per sequence: (round's inputs, row) of every cached token
    for i in range(n_rounds):
        before = srv.lens.tolist()
        x = srv.draw(50 + i)
        srv.lens.add_(srv.runs)
        T().delta_tree_layout(srv.shape, srv.lens, srv.parents, srv.positions, srv.masks, srv.offsets, srv.max_new)
        at = 0
        for b, run in enumerate(x["parents"]):
            depths, sets = sees_of(run)
            rows = slice(at, at + len(run))
            assert srv.positions[rows].tolist() == [before[b] + d for d in depths]
            assert torch.equal(srv.masks[rows].cpu(), mask_words(sets, srv.masks.shape[1]))
            at += len(run)
        srv.lens.sub_(srv.runs)
        srv.round()
        torch.cuda.synchronize()
        at = 0
        for b, (run, n) in enumerate(zip(x["parents"], srv.new)):
            rows = slice(at, at + n)
            want, token = verified(x["target"][rows], x["draft"][rows], x["tokens"][rows], run, x["uniform"][rows])
            assert srv.path[b, :len(want)].tolist() == want and int(srv.n_path[b]) == len(want) and int(srv.next[b]) == token
            assert int(srv.lens[b]) == before[b] + len(want)
            kept[b] += [(x, at + j, before[b] + i) for i, j in enumerate(want)]
            # the accepted rows' attention: all tokens before the run and the accepted ones up to the row
            for layer in range(2):
                k, v = (srv.held(layer, w, b, before[b] + len(want)) for w in range(2))
                for i, j in enumerate(want):
                    m = before[b] + i + 1
                    o, tol = attend(srv.q[layer][at + j].cpu(), k[:m], v[:m], default_scale(HD), P_ROUND)
                    assert worst(srv.out[layer][at + j], o, tol) <= 1, f"round {i}, layer {layer}, row {j} of run {b}"
            at += n
    for b, tokens in enumerate(kept):   # the caches hold the accepted tokens, normed and turned by their place
        for layer in range(2):
            if not tokens:
                continue   # (an empty run)
            k, v = (srv.held(layer, w, b, len(tokens)) for w in range(2))
            raw = torch.stack([x["qkv"][layer][row] for x, row, _ in tokens])
            pos = torch.tensor([p for _, _, p in tokens])
            assert pos.tolist() == list(range(len(tokens)))
            want, tol = turned(*normed(raw[:, HQ:HQ + HKV], srv.weights[1], 1e-6), pos, srv.inv_freq, False)
            for have, w, t, s in ((k, want, tol, 0), (v, raw[:, HQ + HKV:].double(), torch.zeros(1), 1)):
                if srv.scales[layer] is None:
                    half = w.abs() * 2.0 ** -8 if s == 0 else 0.0
                else:
                    unit = srv.scales[layer][s].cpu().double()[:, None]
                    half = torch.maximum(w.abs() * 2.0 ** -4, unit * 2.0 ** -10) * (1 + 2.0 ** -10)
                assert bool(((have - w).abs() <= half + t).all())


def test_rounds_of_drafts():
    check_rounds(Server(), 6)


def test_rounds_of_longer_trees():
    check_rounds(Server(new=(70, 0, 33, 5), capacity=560, seed=3), 3)


def test_captured_rounds_and_two_streams():
    """Two servers, one replaying a captured round and one calling eagerly on a stream of its own, stay alike."""
    a, b = Server(seed=7), Server(seed=7)
    a.draw(1), b.draw(1)
    for s in (a, b):
        s.round()
    torch.cuda.synchronize()
    stream, graph, other = torch.cuda.Stream(), torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        a.round()
    for i in range(5):
        a.draw(10 + i), b.draw(10 + i)
        with torch.cuda.stream(stream):
            graph.replay()
        with torch.cuda.stream(other):
            b.round()
        torch.cuda.synchronize()
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x, y), i


DBG = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                   "paper_2510_09883_amd", "libdelta_attn_debug.so")


@pytest.fixture
def dbg(monkeypatch):
    if not os.path.exists(DBG):
        pytest.skip("the debug library is not built (python -m paper_2510_09883_amd.build --debug)")
    lib = T()._bind(D()._bind(ctypes.CDLL(DBG)))
    monkeypatch.setattr(D(), "_lib", lib)
    return D()


def test_debug_build_gives_the_same_results(dbg):
    check_rounds(Server(seed=8), 3)


@pytest.mark.parametrize("new", [(6, 1, 7), (40, 2, 60)])
def test_debug_build_flags_pages_past_the_cache(dbg, new):
    """The descriptor states fewer pages than the buffers have, so that the bad entry stays inside them: attention
    flags it and reads page 0, append and compaction leave the token out."""
    srv = Server(new=new, seed=9)
    for i in range(3):
        srv.draw(i)
        srv.round()
    torch.cuda.synchronize()
    bad = int(srv.table.max())
    b, page = next((b, p) for b in range(srv.B) for p in range(srv.width) if int(srv.table[b, p]) == bad)
    srv.lens[b] = 16 * page + 3     # the run to come starts in that page
    before = [c[bad].view(torch.uint8).clone() for layer in srv.caches for c in layer]
    for kv in srv.kvs:
        kv.n_pages = bad
    srv.stack = T().CacheStack(srv.shape, srv.kvs)
    srv.ws[:4] = 0
    srv.draw(20)
    srv.round()
    torch.cuda.synchronize()
    if int(srv.lens[b]) <= 16 * srv.width:
        assert int(srv.ws[:4].view(torch.int32)[0]) & dbg.DELTA_DEBUG_PAGE
    after = [c[bad].view(torch.uint8) for layer in srv.caches for c in layer]
    assert all(torch.equal(x, y) for x, y in zip(before, after))


@pytest.mark.parametrize("e4m3", [False, True])
def test_pages_past_32_bits(e4m3):
    """More than 2^32 elements in a cache, pages at both ends: append, attention and compaction."""
    hq, hkv, pages = 16, 8, 262144 + 40     # 2^32 elements are 262144 pages
    kind = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    k, v = (torch.empty((pages, hkv, PAGE, HD), dtype=kind, device="cuda") for _ in range(2))
    table = torch.tensor([[pages - 1, 7, 262144, pages - 3, 131072]], dtype=torch.int32)
    n, m = 75, 45
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    kv = D().make_kv(k, v, table.cuda(), lens)
    shape = D().make_shape(1, hq, hkv, HD, table.shape[1], n)
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((n, hq + 2 * hkv, HD), generator=g).to(torch.bfloat16)
    dev = qkv.cuda()
    q = torch.zeros((n, hq, HD), dtype=torch.bfloat16, device="cuda")
    T().delta_norm_rope_append(shape, kv, dev[:, :hq], dev[:, hq:hq + hkv], dev[:, hq + hkv:], q,
                               row_offsets=offsets_of([n]).cuda())
    place = lambda x, t: x.view(torch.uint8 if e4m3 else torch.int16)[table[0, t // PAGE].long().cuda(), :, (t % PAGE).cuda()]   # noqa: E731
    t = torch.arange(n)
    held = [place(x, t).view(kind).cpu().double() for x in (k, v)]
    assert torch.equal(held[1], qkv[:, hq + hkv:].float().to(kind).double())
    w, part = normed(qkv[:, hq:hq + hkv], None, 1e-6)
    step = torch.maximum(w.abs() * 2.0 ** -4, torch.full((), 2.0 ** -10).double()) if e4m3 else w.abs() * 2.0 ** -8
    assert bool(((held[0] - w).abs() <= step + w.abs() * part).all())
    run = tree(m, "bush", 4)
    sets = sees_of(run)[1]
    out = torch.zeros((m, hq, HD), dtype=torch.bfloat16, device="cuda")
    off = offsets_of([m]).cuda()
    T().delta_tree_attn(shape, kv, q[n - m:].contiguous(), out, mask_words(sets, 2).cuda(), off, m,
                        T().alloc_tree_workspace(shape, m, m))
    torch.cuda.synchronize()
    for j in (0, 9, 30, m - 1):
        seen = list(range(n - m)) + [n - m + i for i in sorted(sets[j])]
        want, tol = attend(q[n - m + j].cpu(), held[0][seen], held[1][seen], default_scale(HD), P_ROUND)
        assert worst(out[j], want, tol) <= 1
    path = torch.tensor([[0, 3, 20, 33, 44]], dtype=torch.int32).cuda()
    new_lens = torch.zeros_like(lens)
    T().delta_cache_compact(T().CacheStack(shape, [kv]), m, off, path, torch.tensor([5], dtype=torch.int32).cuda(), new_lens)
    torch.cuda.synchronize()
    assert int(new_lens) == n - m + 5
    moved = torch.tensor([*range(n - m), *[n - m + i for i in (0, 3, 20, 33, 44)]])
    for x, h in zip((k, v), held):
        assert torch.equal(place(x, torch.arange(n - m + 5)).view(kind).cpu().double(), h[moved])


def test_probabilities_past_32_bits():
    """More than 2^32 values: the last run's rows stand behind them."""
    rows, vocab, n = 30000, 151936, 6
    assert (rows - n) * vocab > 2 ** 32
    target = torch.zeros((rows, vocab), device="cuda")
    g = torch.Generator().manual_seed(5)
    last = torch.softmax(3 * torch.randn((n, vocab), generator=g), -1)
    target[rows - n:] = last.cuda()
    tokens = torch.zeros((rows,), dtype=torch.int32)
    tokens[rows - n + 1:] = last[:-1].argmax(-1).int()
    parents = torch.full((rows,), -1, dtype=torch.int32)
    parents[rows - n:] = torch.tensor([-1, 0, 1, 2, 3, 4], dtype=torch.int32)
    uniform = torch.full((rows,), 0.001)
    uniform[rows - n], uniform[rows - 1] = 0.63, 0.999
    path, n_path, nxt = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((2, n), (2,), (2,)))
    T().delta_verify_drafts(target, None, tokens.cuda(), parents.cuda(), uniform.cuda(),
                            torch.tensor([0, rows - n, rows], dtype=torch.int32).cuda(), path, n_path, nxt,
                            T().alloc_verify_workspace(2, vocab))
    torch.cuda.synchronize()
    want, token = verified(last, None, tokens[rows - n:].tolist(), parents[rows - n:].tolist(), uniform[rows - n:])
    assert path[1, :int(n_path[1])].tolist() == want and len(want) > 1 and int(nxt[1]) == token
    assert n_path[0] == 1 and nxt[0] == -1    # rows of zeros give no token
