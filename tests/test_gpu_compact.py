"""delta_cache_compact against copies on the host: paths of every kind, several layers of both types, and that
nothing else is written."""
import pytest
import torch

from cache_cases import PAGE, Cache
from draft_cases import offsets_of
from gpu_helpers import D

pytestmark = pytest.mark.gpu


def T():
    from paper_2510_09883_amd import drafts
    return drafts


class Call:
    """paths: accepted places per sequence; layers: an e4m3 flag each."""

    def __init__(self, lens, new, paths, hkv=2, d=64, layers=(False,), seed=0, width=None, max_new=None, offsets=True):
        self.lens, self.new, self.paths = lens, new, paths
        self.max_new = max(max(new), 1) if max_new is None else max_new
        self.caches = [Cache([max(s, 1) for s in lens], hkv, d, e4m3=e, seed=seed + i, width=width)
                       for i, e in enumerate(layers)]
        self.seq_lens = torch.tensor(lens, dtype=torch.int32).cuda()
        self.gpu, kvs = [], []
        for c in self.caches:
            self.gpu.append([x.cuda() for x in c.stored])
            sc = {n: s.cuda() for n, s in (("k_scale", c.k_scale), ("v_scale", c.v_scale)) if s is not None}
            kvs.append(D().make_kv(*self.gpu[-1], c.table.cuda(), self.seq_lens, **sc))
        w = self.caches[0].width
        self.shape = D().make_shape(len(lens), 2 * hkv, hkv, d, w, min(max(max(lens), 1), 16 * w))
        self.stack = T().CacheStack(self.shape, kvs)
        path = torch.full((len(lens), self.max_new), -1, dtype=torch.int32)
        for b, p in enumerate(paths):
            path[b, :min(len(p), self.max_new)] = torch.tensor(p[:self.max_new], dtype=torch.int32)
        self.path = path.cuda()
        self.n_path = torch.tensor([len(p) for p in paths], dtype=torch.int32).cuda()
        self.offsets = offsets_of(new).cuda() if offsets else None
        self.new_lens = torch.full((len(lens),), -9, dtype=torch.int32, device="cuda")

    def run(self, new_lens="own"):
        T().delta_cache_compact(self.stack, sum(self.new), self.offsets, self.path, self.n_path,
                                self.new_lens if new_lens == "own" else new_lens)

    def check(self, left=()):
        """left: sequences that stay as they are."""
        torch.cuda.synchronize()
        want_lens = []
        want = [[x.view(torch.uint8 if c.e4m3 else torch.int16).clone() for x in c.stored] for c in self.caches]
        for b, (s, n, p) in enumerate(zip(self.lens, self.new, self.paths)):
            want_lens.append(s if b in left else s - n + len(p))
            if b in left:
                continue
            for to, place in enumerate(p):
                f, t = s - n + place, s - n + to
                for c, layer in zip(self.caches, want):
                    for x in layer:
                        x[int(c.table[b, t // PAGE]), :, t % PAGE] = x[int(c.table[b, f // PAGE]), :, f % PAGE].clone()
        for layer, held in zip(want, self.gpu):
            for w, x in zip(layer, held):
                assert torch.equal(w, x.cpu().view(w.dtype))
        return want_lens


def paths_of(new, seed):
    g = torch.Generator().manual_seed(seed)
    out = []
    for n in new:
        keep = torch.rand((n,), generator=g) < 0.5
        if n:
            keep[0] = True
        out.append(torch.nonzero(keep).flatten().tolist())
    return out


@pytest.mark.parametrize("hkv,d", [(1, 64), (2, 128), (8, 128), (3, 64)])
@pytest.mark.parametrize("layers", [(False,), (True,), (False, True, False)])
def test_accepted_rows_move_together(hkv, d, layers):
    lens = [40, 16, 17, 300, 1, 33, 90]
    new = [7, 16, 1, 40, 1, 0, 64]
    c = Call(lens, new, paths_of(new, hkv), hkv, d, layers, seed=d)
    c.run()
    assert c.new_lens.tolist() == c.check()


def test_paths_of_every_kind():
    """All kept, only the first, only the last, none, neighbours shifted by one, every second."""
    n = 50
    paths = [list(range(n)), [0], [n - 1], [], list(range(1, n)), list(range(0, n, 2)), [0, 1, 2, 30, 31, 49]]
    c = Call([n + 13 * i for i in range(7)], [n] * 7, paths, seed=1)
    c.run()
    assert c.new_lens.tolist() == c.check()


def test_the_longest_runs_and_many_sequences():
    c = Call([512, 700], [512, 500], paths_of([512, 500], 3), seed=2)
    c.run()
    assert c.new_lens.tolist() == c.check()
    new = [b % 6 for b in range(300)]
    c = Call([b % 6 + b % 37 for b in range(300)], new, paths_of(new, 4), seed=3)
    c.run()
    assert c.new_lens.tolist() == c.check()


def test_more_layers_than_a_launch_takes():
    c = Call([30, 9], [9, 4], [[0, 3, 8], [0, 2]], hkv=1, layers=[i % 5 == 0 for i in range(70)], seed=4)
    c.run()
    assert c.new_lens.tolist() == c.check()


@pytest.mark.parametrize("layers", [1, 70])
def test_lengths_in_place_and_not_at_all(layers):
    c = Call([30, 9, 20], [9, 4, 0], [[0, 3, 8], [0, 2], []], hkv=1, layers=[False] * layers, seed=5)
    c.run(None)
    want = c.check()
    assert c.seq_lens.tolist() == c.lens and c.new_lens.tolist() == [-9] * 3
    c = Call([30, 9, 20], [9, 4, 0], [[0, 3, 8], [0, 2], []], hkv=1, layers=[False] * layers, seed=5)
    c.run(c.seq_lens)
    c.check()
    assert c.seq_lens.tolist() == want


@pytest.mark.parametrize("in_place", [False, True])
def test_paths_that_are_none_leave_a_sequence_alone(in_place):
    """Not ascending, twice the same, past the run, negative, more than the run; a run that does not fit."""
    n = 8
    paths = [[0, 3, 2], [0, 2, 2], [0, 8], [-1, 2], list(range(9)), [0, 5], [0, 3]]
    lens = [40, 41, 42, 43, 44, 5, 45]
    c = Call(lens, [n] * 7, paths, seed=6, max_new=n)
    c.n_path[4] = 9
    c.run(c.seq_lens if in_place else "own")
    want = c.check(left=range(6))
    assert (c.seq_lens if in_place else c.new_lens).tolist() == want
    c = Call([40, 33, 30], [4, 4, 4], [[0, 2], [0, 2], [0, 3]], seed=7, width=3)
    c.lens[1] = 49   # three pages hold 48
    c.seq_lens[1] = 49
    c.run()
    assert c.new_lens.tolist() == c.check(left=[1])


def test_single_rows_without_offsets():
    c = Call([30, 9, 1], [1, 1, 1], [[0], [], [0]], seed=8, offsets=False)
    c.run()
    assert c.new_lens.tolist() == c.check()


def test_captured_and_replayed():
    c = Call([60, 40], [20, 16], [[0, 2, 9, 15], [0, 4]], hkv=2, d=128, layers=(False, True), seed=9)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        c.run(c.seq_lens)
    for paths in ([[0, 2, 9, 15], [0, 4]], [[0], [1, 2, 3]], [[0, 1, 2], list(range(0, 16, 3))]):
        c.paths = paths
        c.path.fill_(-1)
        for b, p in enumerate(paths):
            c.path[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
        c.n_path.copy_(torch.tensor([len(p) for p in paths], dtype=torch.int32))
        c.seq_lens.copy_(torch.tensor(c.lens, dtype=torch.int32))
        for layer, cache in zip(c.gpu, c.caches):
            for x, s in zip(layer, cache.stored):
                x.copy_(s)
        torch.cuda.synchronize()
        graph.replay()
        want = c.check()
        assert c.seq_lens.tolist() == want


def test_refusals():
    c = Call([30, 9], [9, 4], [[0, 3, 8], [0, 2]], layers=(False, True), seed=10)
    err = D().DeltaError

    def call(error, match, stack=c.stack, n=13, off=c.offsets, path=c.path, n_path=c.n_path, lens=c.new_lens):
        with pytest.raises(error, match=match):
            T().delta_cache_compact(stack, n, off, path, n_path, lens)
    call(ValueError, "^path: expected shape", path=c.path[:1])
    call(ValueError, "^path: expected torch.int32", path=c.path.long())
    call(ValueError, "^n_path: expected", n_path=c.n_path[:1])
    call(ValueError, "^new_lens: expected", lens=c.new_lens[:1])
    call(ValueError, "^row_offsets", off=c.offsets[:2])
    call(err, "invalid argument", off=None)
    call(err, "invalid argument", n=8)          # runs of 9 of 8 rows
    call(err, "invalid argument", n=-1)
    k, v = c.gpu[0]
    other = D().make_kv(k, v, c.caches[0].table.cuda(), c.seq_lens.clone())
    call(err, "invalid argument", stack=T().CacheStack(c.shape, [c.stack.layers[0], other]))
    with pytest.raises(ValueError, match="at least one layer"):
        T().CacheStack(c.shape, [])
    with pytest.raises(ValueError, match="^k_cache: expected shape"):
        T().CacheStack(D().make_shape(2, 8, 4, 64, c.caches[0].width, 30), c.stack.layers)
    torch.cuda.synchronize()
    c.paths, c.new = [[], []], [0, 0]
    c.check()
    assert c.new_lens.tolist() == [-9, -9]
