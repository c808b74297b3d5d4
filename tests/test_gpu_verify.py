"""delta_verify_drafts against the definition in exact arithmetic: chains and trees, drawn and chosen drafts,
borders that are met exactly, distributions with holes, and odd sizes of everything."""
import pytest
import torch

from draft_cases import offsets_of, tree, verified
from gpu_helpers import D

pytestmark = pytest.mark.gpu


def T():
    from paper_2510_09883_amd import drafts
    return drafts


class Call:
    """Runs of trees with probabilities of a target and (drawn) of a drafting model near it."""

    def __init__(self, new, vocab, kind="bush", drawn=False, seed=0, pad=0, max_new=None, sharp=1.5, gap=0,
                 offsets=True):
        g = torch.Generator().manual_seed(seed)
        self.new, self.vocab = new, vocab
        rows = sum(new) + pad
        logits = torch.randn((rows, vocab), generator=g) * sharp
        near = logits + 0.7 * torch.randn((rows, vocab), generator=g)
        self.target = torch.softmax(logits, -1)
        self.draft = torch.softmax(near, -1) if drawn else None
        self.parents = [p for b, n in enumerate(new) for p in tree(n, kind, seed + b)] + [0] * pad
        self.tokens, at = [], 0
        for n in new:
            for j in range(n):
                p = max(self.parents[at + j], 0)
                if drawn:
                    self.tokens.append(int(torch.multinomial(self.draft[at + p], 1, generator=g)))
                else:
                    self.tokens.append(int(near[at + p].topk(min(vocab, 1 + j % 4)).indices[-1]))
            at += n
        self.tokens += [0] * pad
        self.uniform = torch.rand((rows,), generator=g)
        self.max_new = max(max(new), 1) if max_new is None else max_new
        self.offsets, self.gap = offsets, gap

    def run(self, ws=None):
        """The call's outputs (path, n_path, next); rows `gap` values apart."""
        rows, B = self.target.shape[0], len(self.new)

        def rowwise(t):
            if t is None:
                return None
            wide = torch.full((rows, self.vocab + self.gap), float("nan"), device="cuda")
            wide[:, :self.vocab] = t.cuda()
            return wide[:, :self.vocab]
        i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()   # noqa: E731
        out = [torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((B, self.max_new), (B,), (B,))]
        self.ws = T().alloc_verify_workspace(B, self.vocab) if ws is None else ws
        T().delta_verify_drafts(rowwise(self.target), rowwise(self.draft), i32(self.tokens), i32(self.parents),
                                self.uniform.cuda(), offsets_of(self.new).cuda() if self.offsets else None, *out, self.ws)
        torch.cuda.synchronize()
        return [x.cpu() for x in out]

    def check(self, ws=None):
        path, n_path, nxt = self.run(ws)
        at = 0
        accepted = 0
        for b, n in enumerate(self.new):
            rows = slice(at, at + n)
            want, token = verified(self.target[rows], None if self.draft is None else self.draft[rows],
                                   self.tokens[rows], self.parents[rows], self.uniform[rows])
            have = path[b, :int(n_path[b])].tolist()
            assert have == want, f"path of run {b}"
            assert bool((path[b, len(want):] == -1).all())
            assert int(nxt[b]) == token, f"token after run {b}"
            accepted += max(0, len(want) - 1)
            at += n
        return accepted


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("kind", ["chain", "star", "pairs", "bush"])
@pytest.mark.parametrize("vocab", [2, 37, 300])
def test_trees(vocab, kind, drawn):
    accepted = 0
    for seed in range(3):
        accepted += Call([5, 0, 1, 12, 33, 3], vocab, kind, drawn, seed=seed, pad=2).check()
    assert accepted > 0   # (some drafts stand)


@pytest.mark.parametrize("drawn", [False, True])
def test_large_vocabularies(drawn):
    """Several pieces a row, the last one partial, rows that start at any 4 bytes."""
    for vocab, gap in ((2049, 0), (5003, 2), (16385, 1)):
        Call([4, 2, 7], vocab, "bush", drawn, seed=vocab, gap=gap, sharp=3.0).check()


def test_the_whole_vocabulary_is_reached():
    """u0 walks the unit interval: every piece and window gives its tokens."""
    vocab = 9001
    c = Call([1] * 60, vocab, seed=3, sharp=1.0)
    c.uniform = torch.arange(60) / 60.0
    c.check()
    c.uniform[:] = 1.0 - 2.0 ** -24
    c.check()
    c.uniform[:] = 0.0
    c.check()


def test_one_sequence_and_many():
    Call([1], 64, seed=1).check()
    Call([9], 20000, "bush", True, seed=2).check()
    Call([(b * 7) % 4 for b in range(1500)], 40, "bush", True, seed=3).check()
    Call([2] * 70, 700, "chain", seed=4, max_new=5).check()


def test_single_rows_without_offsets():
    c = Call([1] * 5, 100, seed=5, offsets=False)
    c.check()


@pytest.mark.parametrize("drawn", [False, True])
def test_the_longest_runs(drawn):
    for kind in ("chain", "star", "bush"):
        c = Call([512, 130], 6 if kind == "chain" else 40, kind, drawn, seed=7)
        if kind == "chain":   # the drafts are what the target would say: long paths
            for b, (at, n) in enumerate(((0, 512), (512, 130))):
                for j in range(1, n):
                    c.tokens[at + j] = int(c.target[at + j - 1].argmax())
                c.target[at:at + n] = torch.softmax(6 * c.target[at:at + n].log(), -1)
                if drawn:
                    c.draft[at:at + n] = c.target[at:at + n]
        c.check()


def test_borders_that_are_met_exactly():
    """Multiples of 2^-6: sums and products are exact in 64 bits.  u q = p is a rejection, and a partial sum of
    exactly u0 times the whole is not passed."""
    p = torch.tensor([[8, 0, 24, 32], [16, 16, 16, 16], [0, 0, 0, 64]], dtype=torch.float32) / 64
    q = torch.tensor([[32, 16, 8, 8], [64, 0, 0, 0], [16, 16, 16, 16]], dtype=torch.float32) / 64

    def one(u, tokens, draft):
        c = Call([3], 4)
        c.target, c.draft, c.parents, c.tokens, c.uniform = p, draft, [-1, 0, 1], tokens, torch.tensor(u)
        path, n, nxt = c.run()
        c.check()
        return path[0].tolist(), int(nxt)
    assert one([0.5, 0.25, 0.5], [0, 0, 0], q)[0] == [0, -1, -1]      # 0.25 * 0.5 = 0.125: rejected
    assert one([0.5, 0.2499, 0.25], [0, 0, 0], q)[0] == [0, 1, -1]    # accepted; then 0.25 * 1 = 0.25: rejected
    assert one([0.5, 0.2499, 0.2499], [0, 0, 0], q) == ([0, 1, 2], 3)
    assert one([0.5, 0.125, 0.9], [0, 0, 0], None)[0] == [0, -1, -1]  # u = p
    # after the rejection of token 0: 24 and 32 of 56 are left, u0 = 3/7 is not exact, 0 and 24/64 are
    assert one([0.0, 0.125, 0.9], [0, 0, 0], None) == ([0, -1, -1], 2)
    c = Call([1], 4)
    c.target, c.uniform, c.tokens, c.parents = p[:1], torch.tensor([0.125]), [0], [-1]
    assert c.run()[2].tolist() == [2]       # the partial sum 8/64 is met, not passed; token 1 has no probability
    c.uniform = torch.tensor([0.5])
    assert c.run()[2].tolist() == [3]


def test_greedy_targets():
    """Distributions of one token: drafts stand exactly where they agree."""
    new, vocab = [6, 4], 5000
    c = Call(new, vocab, "chain", seed=8)
    best = torch.randint(0, vocab, (10,), generator=torch.Generator().manual_seed(1))
    c.target = torch.nn.functional.one_hot(best, vocab).float()
    c.tokens = [0, *best[:3].tolist(), 4999, 7, 0, *best[6:9].tolist()]
    path, n, nxt = c.run()
    c.check()
    assert n.tolist()[1] == 4 and nxt.tolist()[1] == int(best[9])


def test_equal_distributions_accept_all():
    for drawn in (True,):
        c = Call([8, 3], 200, "chain", drawn, seed=9)
        c.draft = c.target.clone()
        path, n, _ = c.run()
        c.check()
        assert n.tolist() == [8, 3]     # u < 1


def test_siblings_with_the_same_token():
    for drawn in (False, True):
        c = Call([7, 40], 12, "star", drawn, seed=10)
        c.tokens = [t % 3 for t in c.tokens]
        c.uniform[1:] = c.uniform[1:].clamp(min=0.6)
        c.check()


def test_residuals_of_nothing():
    """p below q everywhere it could be drawn: after the rejection nothing is left, and p takes its place; rows of
    zeros give no token."""
    c = Call([2, 2, 1], 6, "chain", True, seed=11)
    c.target[0] = c.draft[0] * 0.5
    c.uniform[1] = 0.9
    c.tokens[1] = int(c.draft[0].argmax())
    c.target[2] = 0.0
    c.target[4] = 0.0
    path, n, nxt = c.run()
    c.check()
    assert n.tolist() == [1, 1, 1] and nxt.tolist()[1:] == [-1, -1]
    c = Call([4], 5, "star", False, seed=12)    # all tokens with probability are rejected
    c.target[0] = torch.tensor([0.25, 0.25, 0.5, 0, 0])
    c.tokens, c.uniform = [0, 0, 1, 2], torch.tensor([0.6, 0.9, 0.9, 0.99])
    c.check()


def test_tokens_and_parents_that_name_nothing_and_odd_values():
    c = Call([6, 6], 50, "star", seed=13)
    c.tokens[1], c.tokens[2], c.tokens[3] = -1, 50, 2 ** 31 - 1
    c.parents[4] = -1                      # never tried
    c.parents[9], c.parents[10] = 9, 11    # itself, a later one
    c.target[0, 3] = float("nan")
    c.target[6, 7] = -0.25
    c.check()
    c = Call([6, 6], 50, "star", True, seed=14)
    c.target[0, 3], c.draft[0, 4], c.draft[6, :9] = float("nan"), float("nan"), 0.0
    c.tokens[1], c.tokens[2], c.tokens[8] = -1, 50, 4
    c.check()


def test_longer_runs_than_stated_are_cut():
    c = Call([9, 3], 80, "chain", seed=15, max_new=4)
    path, n, _ = c.run()
    assert int(n.max()) <= 4
    cut = Call([9, 3], 80, "chain", seed=15)
    at = 0
    for b, m in enumerate((9, 3)):
        m4 = min(m, 4)
        want, _ = verified(cut.target[at:at + m4], None, cut.tokens[at:at + m4], cut.parents[at:at + m4],
                           cut.uniform[at:at + m4])
        assert path[b, :int(n[b])].tolist() == want
        at += m


def test_equal_calls_a_shared_workspace_and_graph_replays():
    ws = T().alloc_verify_workspace(40, 30000)
    a = Call([5] * 40, 900, "bush", True, seed=16)
    b = Call([3, 9], 30000, "bush", seed=17, sharp=3.0)
    for _ in range(2):   # every call leaves the workspace ready for the next, of any size
        a.check(ws)
        b.check(ws)
    first = a.run(ws)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()   # noqa: E731
    args = [a.target.cuda(), a.draft.cuda(), i32(a.tokens), i32(a.parents), a.uniform.cuda(), offsets_of(a.new).cuda()]
    out = [torch.zeros_like(x).cuda() for x in first]
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        T().delta_verify_drafts(*args, *out, ws)
    for _ in range(4):
        for x in out:
            x.fill_(-9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x.cpu(), w) for x, w in zip(out, first))
        b.check(ws)


def test_refusals():
    c = Call([2, 3], 40, drawn=True, seed=18)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()   # noqa: E731
    good = dict(target=c.target.cuda(), draft=c.draft.cuda(), tokens=i32(c.tokens), parents=i32(c.parents),
                uniform=c.uniform.cuda(), off=offsets_of(c.new).cuda(), path=i32([[0] * 3] * 2), n=i32([7, 7]),
                nxt=i32([7, 7]), ws=T().alloc_verify_workspace(2, 40))
    err = D().DeltaError

    def call(error, match, **kw):
        a = {**good, **kw}
        with pytest.raises(error, match=match):
            T().delta_verify_drafts(a["target"], a["draft"], a["tokens"], a["parents"], a["uniform"], a["off"],
                                    a["path"], a["n"], a["nxt"], a["ws"])
    call(ValueError, "^target: expected torch.float32", target=good["target"].double())
    call(ValueError, "^target: must be a GPU", target=c.target)
    call(ValueError, "one behind the other", target=good["target"].t().contiguous().t())
    call(ValueError, "^draft: expected shape", draft=good["draft"][:, :39].contiguous())
    call(ValueError, "^tokens: expected", tokens=good["tokens"].long())
    call(ValueError, "^uniform: expected", uniform=good["uniform"][:4])
    call(ValueError, "^row_offsets: expected", off=good["off"][:2])
    call(ValueError, "^n_path: expected", n=good["n"][:1])
    call(err, "invalid argument", off=None)
    call(err, "invalid argument", path=i32([[0] * 6] * 2))          # runs of 6 of 5 rows
    call(err, "invalid argument", target=good["target"].expand(5, 40)[:1].expand(5, 40), draft=None)   # rows on one another
    call(err, "workspace too small", ws=good["ws"][:256])
    call(err, "invalid argument", ws=torch.zeros(9000, dtype=torch.uint8, device="cuda")[8:])
    torch.cuda.synchronize()
    assert good["n"].tolist() == [7, 7] and not good["path"].any()
    with pytest.raises(err, match="unsupported"):
        T().alloc_verify_workspace(2, (1 << 20) + 1)
