"""delta_rope_append against the rotation in float64: ragged runs, both pairings, partly rotated heads,
far positions, strided inputs, both cache types, and that nothing else is written."""
import ctypes

import pytest
import torch

from cache_cases import PAGE, Cache
from gpu_helpers import D

pytestmark = pytest.mark.gpu


def E():
    from paper_2510_09883_amd import extend
    return extend


def frequencies(rot, base=10000.0):
    return (base ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))).float()


def rotated(x, pos, inv_freq, interleaved):
    """float64 rotation of [rows, heads, d], and how far fp32 arithmetic may be off: each of two
    products and their sum 2^-24, sine and cosine 2^-22 (angle reduced in fp64, then rounded)."""
    n = inv_freq.numel()
    w = x.double().clone()
    if n == 0:
        return w, torch.zeros_like(w)
    a = pos.double()[:, None, None] * inv_freq.double()
    i, j = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    p, r = w[..., i].clone(), w[..., j].clone()
    w[..., i], w[..., j] = p * a.cos() - r * a.sin(), r * a.cos() + p * a.sin()
    tol = torch.zeros_like(w)
    tol[..., i] = tol[..., j] = (p.abs() + r.abs()) * 2.0 ** -21
    return w, tol


class Call:
    """A call's tensors on the GPU and what it has to leave behind."""

    def __init__(self, lens, new, hq, hkv, d, rot, e4m3=False, scales=True, interleaved=False, packed=True,
                 pad=0, seed=0, positions=False, inv_freq=None, offsets=True, width=None, with_q=True):
        g = torch.Generator().manual_seed(seed)
        self.cache = Cache([max(s, 1) for s in lens], hkv, d, e4m3=e4m3, scales=scales, seed=seed, width=width)
        self.lens, self.new, self.dims = lens, new, (hq, hkv, d)
        self.rows = sum(new) + pad
        self.interleaved = interleaved
        self.inv_freq = frequencies(rot) if inv_freq is None else inv_freq
        qkv = torch.randn((self.rows, hq + 2 * hkv, d), generator=g).to(torch.bfloat16)
        self.q, self.k, self.v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        dev = qkv.cuda()
        self.gpu = [dev[:, :hq], dev[:, hq:hq + hkv], dev[:, hq + hkv:]]
        if not packed:
            self.gpu = [t.contiguous() for t in self.gpu]
        self.positions = torch.randint(0, 5000, (self.rows,), generator=g).int() if positions else None
        self.offsets = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32).cuda() if offsets else None
        self.table = self.cache.table.cuda()
        self.seq_lens = torch.tensor(lens, dtype=torch.int32).cuda()
        self.kv_gpu = [x.cuda() for x in self.cache.stored]
        sc = {n: s.cuda() for n, s in (("k_scale", self.cache.k_scale), ("v_scale", self.cache.v_scale)) if s is not None}
        self.kv = D().make_kv(self.kv_gpu[0], self.kv_gpu[1], self.table, self.seq_lens, **sc)
        self.shape = D().make_shape(len(lens), hq, hkv, d, self.cache.width, min(max(max(lens), 1), 16 * self.cache.width))
        self.out = torch.full((self.rows, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
        self.with_q = with_q

    def run(self):
        f = self.inv_freq.cuda() if self.inv_freq.numel() else None
        p = self.positions.cuda() if self.positions is not None else None
        q = (self.gpu[0], self.out) if self.with_q else (None, None)
        E().delta_rope_append(self.shape, self.kv, q[0], self.gpu[1], self.gpu[2], q[1], f,
                              row_offsets=self.offsets, positions=p, interleaved=self.interleaved)

    def check(self):
        torch.cuda.synchronize()
        hq, hkv, d = self.dims
        e4m3 = self.cache.e4m3
        want = [x.clone() for x in self.cache.stored]
        raw = [x.view(torch.uint8 if e4m3 else torch.int16) for x in want]
        got = [x.cpu() for x in self.kv_gpu]
        q_left = torch.ones(self.rows, dtype=torch.bool)
        row = 0
        for b, (s, n) in enumerate(zip(self.lens, self.new)):
            rows = slice(row, row + n)
            row += n
            if s < n or s > 16 * self.cache.width:
                continue   # a run without room is skipped
            q_left[rows] = not self.with_q
            t = torch.arange(s - n, s)
            pos = t if self.positions is None else self.positions[rows].long()
            if self.with_q:
                w, tol = rotated(self.q[rows], pos, self.inv_freq, self.interleaved)
                off = (self.out[rows].double().cpu() - w).abs()
                assert bool((off <= tol + w.abs() * 2.0 ** -8).all()), f"queries of run {b}"
            page, at = self.cache.table[b, t // PAGE].long(), t % PAGE
            for which, x in ((0, self.k), (1, self.v)):
                w, tol = rotated(x[rows], pos, self.inv_freq, self.interleaved) if which == 0 else \
                    (x[rows].double(), torch.zeros(1, dtype=torch.float64))
                have = got[which][page, :, at].double()
                if e4m3:
                    scale = (self.cache.k_scale, self.cache.v_scale)[which]
                    if scale is not None:
                        w, tol = w / scale.double()[:, None], tol / scale.double()[:, None]
                    w = w.clamp(-448, 448)
                    # half a step: 2^-4 of the value, 2^-10 below 2^-6; the quotient's own rounding
                    tol = tol + torch.clamp(w.abs() * 2.0 ** -4, min=2.0 ** -10) + w.abs() * 2.0 ** -23
                else:
                    tol = tol + (w.abs() * 2.0 ** -8 if which == 0 else 0.0)
                assert bool(((have - w).abs() <= tol).all()), f"{'KV'[which]} of run {b}"
                raw[which][page, :, at] = got[which].view(raw[which].dtype)[page, :, at]
        for w, x in zip(raw, got):   # every other row of the caches is what it was, bit for bit
            assert torch.equal(w, x.view(w.dtype))
        assert bool((self.out[q_left.cuda()] == 7.0).all())


RUNS = [([1], [1]), ([40], [40]), ([5, 16, 17, 300], [0, 16, 1, 299]), ([33, 1, 2, 64, 500], [33, 1, 2, 3, 0])]


@pytest.mark.parametrize("lens,new", RUNS)
@pytest.mark.parametrize("hq,hkv,d,rot,inter", [(8, 2, 64, 64, False), (28, 4, 128, 128, False), (3, 3, 64, 16, True),
                                                (10, 2, 128, 64, False), (8, 1, 128, 128, True), (4, 4, 128, 48, True)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_rows_match_float64(lens, new, hq, hkv, d, rot, inter, e4m3):
    c = Call(lens, new, hq, hkv, d, rot, e4m3=e4m3, interleaved=inter, pad=3, seed=len(lens) + d)
    c.run()
    c.check()


@pytest.mark.parametrize("e4m3,packed", [(False, False), (True, True)])
def test_many_sequences_single_tokens_and_explicit_positions(e4m3, packed):
    lens = [(13 * b) % 90 + 1 for b in range(150)]
    for offsets in (True, False):
        c = Call(lens, [1] * 150, 12, 2, 128, 128, e4m3=e4m3, packed=packed, seed=4, positions=offsets,
                 offsets=offsets)
        c.run()
        c.check()
    c = Call([0, 3] * 70 + [0], [0, 2] * 70 + [0], 4, 2, 64, 64, e4m3=e4m3, packed=packed, seed=5, pad=1)
    c.run()
    c.check()


@pytest.mark.parametrize("batch", [64, 65, 300, 4097])
def test_rows_are_found_among_many_sequences(batch):
    """Empty runs between others, at every size of the search for a row's sequence."""
    new = [(b * 7 + 1) % 3 for b in range(batch)]
    c = Call([n + b % 5 for b, n in enumerate(new)], new, 2, 1, 64, 16, seed=batch, pad=2)
    c.run()
    c.check()


def test_large_prompts_share_workgroups():
    """Few heads and many rows: several rows a workgroup, the last one partly filled."""
    c = Call([4500, 600], [4500, 599], 2, 1, 64, 64, seed=15, pad=3)
    c.run()
    c.check()


@pytest.mark.parametrize("base", [1.0, 10000.0, 1e6])
def test_far_positions(base):
    """Angles up to 131071 radians: an fp32 angle would be off by 0.004."""
    s = 131071
    c = Call([s], [5], 4, 1, 128, 128, seed=6, inv_freq=frequencies(128, base))
    c.run()
    c.check()


def test_without_rotation_and_without_queries():
    for e4m3 in (False, True):
        c = Call([40, 7], [30, 7], 8, 2, 128, 128, e4m3=e4m3, scales=False, seed=7, with_q=False,
                 inv_freq=torch.zeros(0))
        c.run()
        c.check()


def test_runs_without_room_are_skipped():
    """A length below the run's, a length past the page table: nothing of that run is written."""
    c = Call([20, 3, 33, 10], [4, 5, 2, 10], 8, 2, 64, 64, seed=8, width=3)
    c.lens[2] = 49   # three pages hold 48
    c.seq_lens[2] = 49
    c.run()
    c.check()


def test_rotated_in_place():
    c = Call([30, 9], [12, 9], 8, 2, 128, 128, packed=False, seed=9)
    c.out = c.gpu[0]
    c.run()
    torch.cuda.synchronize()
    c.check()


def test_saturation_and_nan_in_an_e4m3_cache():
    c = Call([16], [16], 2, 1, 64, 16, e4m3=True, scales=False, seed=10, inv_freq=torch.zeros(0))
    x = torch.tensor([0.0, -0.0, 447.0, 448.0, 463.9, 465.0, 1e4, float("inf"), -1e4, float("-inf"),
                      float("nan"), 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -11, 2.0 ** -11, -1.0625])
    c.gpu[1][0, 0, :16] = x.cuda().to(torch.bfloat16)
    c.gpu[2][3, 0, 16:32] = x.cuda().to(torch.bfloat16)
    c.run()
    torch.cuda.synchronize()
    want = x.to(torch.bfloat16).float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    page = int(c.cache.table[0, 0])
    for got in (c.kv_gpu[0][page, 0, 0, :16], c.kv_gpu[1][page, 0, 3, 16:32]):
        got = got.cpu().view(torch.uint8)
        nan = x.isnan()
        assert bool(((got & 0x7F) == 0x7F)[nan].all()) and torch.equal(got[~nan], want[~nan])


def test_replays_and_another_stream():
    """Captured once; replayed with new inputs and other lengths, on a stream of its own."""
    c = Call([40, 17, 64], [9, 17, 1], 12, 2, 128, 128, e4m3=True, seed=11)
    f = c.inv_freq.cuda()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        E().delta_rope_append(c.shape, c.kv, c.gpu[0], c.gpu[1], c.gpu[2], c.out, f, row_offsets=c.offsets)
    for seed, lens in ((1, [40, 17, 64]), (2, [33, 20, 10]), (3, [9, 30, 64])):
        torch.cuda.synchronize()
        g = torch.Generator().manual_seed(seed)
        x = torch.randn((c.rows, 16, 128), generator=g).to(torch.bfloat16)
        for i, part in enumerate((x[:, :12], x[:, 12:14], x[:, 14:])):
            c.gpu[i].copy_(part)
        c.q, c.k, c.v = x[:, :12], x[:, 12:14], x[:, 14:]
        c.lens = lens
        c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        for t, s in zip(c.kv_gpu, c.cache.stored):
            t.copy_(s)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        c.check()


def test_no_rows():
    c = Call([5, 9], [0, 0], 8, 2, 64, 64, seed=12)
    c.run()
    c.check()


def test_refusals():
    c = Call([20, 30], [2, 3], 8, 2, 64, 64, seed=13)
    q, k, v = c.gpu
    f = c.inv_freq.cuda()

    def call(error, match, **kw):
        a = dict(q=q, k=k, v=v, out=c.out, f=f, off=c.offsets, pos=None)
        a.update(kw)
        with pytest.raises(error, match=match):
            E().delta_rope_append(c.shape, c.kv, a["q"], a["k"], a["v"], a["out"], a["f"], row_offsets=a["off"],
                                  positions=a["pos"])
    call(ValueError, "^k: expected shape", k=k[:, :1])
    call(ValueError, "^v: 4 rows", v=v[:4])
    call(ValueError, "^q: 4 rows", q=q[:4])
    call(ValueError, "^q: expected torch.bfloat16", q=q.float())
    call(ValueError, "^k: must be a GPU", k=c.k)
    call(ValueError, "one behind the other", v=v.transpose(1, 2).contiguous().transpose(1, 2))
    call(ValueError, "come together", q=None)
    call(ValueError, "^q_out: must be contiguous", out=torch.empty((5, 8, 128), dtype=torch.bfloat16, device="cuda")[..., ::2])
    call(ValueError, "^row_offsets: expected shape", off=c.offsets[:2])
    call(ValueError, "^positions: expected", pos=torch.zeros(5, device="cuda"))
    call(ValueError, "^positions: nothing", f=None, pos=torch.zeros(5, dtype=torch.int32, device="cuda"))
    call(ValueError, "^inv_freq: expected", f=f.double())
    err = D().DeltaError
    call(err, "invalid argument", f=f[:3].contiguous())               # 6 rotated elements
    call(err, "invalid argument", f=torch.ones(40, device="cuda"))    # 80 of 64
    call(err, "invalid argument", off=None)                           # 5 rows of 2 single tokens
    wide = torch.zeros((5, 12 * 64 + 4), dtype=torch.bfloat16, device="cuda")
    call(err, "invalid argument", q=wide[:, :512].view(5, 8, 64))     # a row stride that is not 16 bytes
    call(err, "invalid argument", k=torch.zeros((5 * 128 + 8,), dtype=torch.bfloat16, device="cuda")[4:644].view(5, 2, 64))
    torch.cuda.synchronize()
    c.lens, c.new = [20, 30], [0, 0]
    c.check()   # nothing was written
    rope = E().delta_rope_t(f.data_ptr(), None, 64, 2)
    assert D()._lib.delta_rope_append(ctypes.byref(c.shape), ctypes.byref(c.kv), ctypes.byref(rope), 5,
                                      c.offsets.data_ptr(), None, 0, k.data_ptr(), 768, v.data_ptr(), 768,
                                      None, None) == -1
