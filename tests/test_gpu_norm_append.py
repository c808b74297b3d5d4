"""delta_norm_rope_append against the norm and the rotation in float64: weights of both types and none,
ragged runs, both pairings, partly rotated heads, positions, strided inputs, both cache types, and that
nothing else is written."""
import ctypes

import pytest
import torch

from cache_cases import PAGE
from gpu_helpers import D
from test_gpu_rope_append import Call as RopeCall
from test_gpu_rope_append import frequencies

pytestmark = pytest.mark.gpu


def T():
    from paper_2510_09883_amd import drafts
    return drafts


def normed(x, weight, eps):
    """float64 norm of [rows, heads, d], and the part of each value that fp32 arithmetic may be off: the sum of
    d squares by d + 1 roundings of 2^-24, of which the root takes half; a root, a quotient and two products
    by 2^-22 together with room for one more."""
    w = torch.ones(x.shape[-1], dtype=torch.float64) if weight is None else weight.double()
    y = x.double() / (x.double().square().mean(-1, keepdim=True) + eps).sqrt() * w
    return y, (x.shape[-1] + 1) / 2 * 2.0 ** -24 + 2.0 ** -21


def turned(y, part, pos, inv_freq, interleaved):
    """float64 rotation of normed heads and how far fp32 may be off (see test_gpu_rope_append.rotated)."""
    n = inv_freq.numel()
    w, tol = y.clone(), y.abs() * part
    if n:
        a = pos.double()[:, None, None] * inv_freq.double()
        i, j = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
        p, r = y[..., i], y[..., j]
        w[..., i], w[..., j] = p * a.cos() - r * a.sin(), r * a.cos() + p * a.sin()
        tol[..., i] = tol[..., j] = (p.abs() + r.abs()) * (2.0 ** -21 + part)
    return w, tol


class Call(RopeCall):
    def __init__(self, *args, weights="bf16", eps=1e-6, gain=1.0, **kw):
        super().__init__(*args, **kw)
        g = torch.Generator().manual_seed(77)
        d = self.dims[2]
        self.eps = eps
        self.weights = [None, None]
        if weights != "none":
            w = 1.0 + 0.3 * torch.randn((2, d), generator=g)
            w = w if weights == "f32" else w.to(torch.bfloat16)
            self.weights = [w[0], None if weights == "q" else w[1]]
        for t, dev in zip((self.q, self.k), self.gpu):
            t.mul_(gain)
            dev.copy_(t)

    def run(self):
        f = self.inv_freq.cuda() if self.inv_freq.numel() else None
        p = self.positions.cuda() if self.positions is not None else None
        q = (self.gpu[0], self.out) if self.with_q else (None, None)
        w = [None if x is None else x.cuda().contiguous() for x in self.weights]
        T().delta_norm_rope_append(self.shape, self.kv, q[0], self.gpu[1], self.gpu[2], q[1], w[0], w[1], self.eps, f,
                                   row_offsets=self.offsets, positions=p, interleaved=self.interleaved)

    def check(self):
        torch.cuda.synchronize()
        e4m3 = self.cache.e4m3
        raw = [x.clone().view(torch.uint8 if e4m3 else torch.int16) for x in self.cache.stored]
        got = [x.cpu() for x in self.kv_gpu]
        q_left = torch.ones(self.rows, dtype=torch.bool)
        row = 0
        for b, (s, n) in enumerate(zip(self.lens, self.new)):
            rows = slice(row, row + n)
            row += n
            if s < n or s > 16 * self.cache.width or n == 0:
                continue   # a run without room is skipped
            q_left[rows] = not self.with_q
            t = torch.arange(s - n, s)
            pos = t if self.positions is None else self.positions[rows].long()
            if self.with_q:
                w, tol = turned(*normed(self.q[rows], self.weights[0], self.eps), pos, self.inv_freq, self.interleaved)
                off = (self.out[rows].double().cpu() - w).abs()
                assert bool((off <= tol + w.abs() * 2.0 ** -8).all()), f"queries of run {b}"
            page, at = self.cache.table[b, t // PAGE].long(), t % PAGE
            for which in (0, 1):
                if which == 0:
                    w, tol = turned(*normed(self.k[rows], self.weights[1], self.eps), pos, self.inv_freq,
                                    self.interleaved)
                else:
                    w, tol = self.v[rows].double(), torch.zeros(1, dtype=torch.float64)
                have = got[which][page, :, at].double()
                if e4m3:
                    scale = (self.cache.k_scale, self.cache.v_scale)[which]
                    if scale is not None:
                        w, tol = w / scale.double()[:, None], tol / scale.double()[:, None]
                    w = w.clamp(-448, 448)
                    tol = tol + torch.clamp(w.abs() * 2.0 ** -4, min=2.0 ** -10) + w.abs() * 2.0 ** -23
                else:
                    tol = tol + (w.abs() * 2.0 ** -8 if which == 0 else 0.0)
                assert bool(((have - w).abs() <= tol).all()), f"{'KV'[which]} of run {b}"
                raw[which][page, :, at] = got[which].view(raw[which].dtype)[page, :, at]
        for w, x in zip(raw, got):   # every other row of the caches is what it was, bit for bit
            assert torch.equal(w, x.view(w.dtype))
        assert bool((self.out[q_left.cuda()] == 7.0).all())


RUNS = [([1], [1]), ([5, 16, 17, 300], [0, 16, 1, 299]), ([33, 1, 2, 64, 500], [33, 1, 2, 3, 0])]


@pytest.mark.parametrize("lens,new", RUNS)
@pytest.mark.parametrize("hq,hkv,d,rot,inter,weights", [
    (8, 2, 64, 64, False, "bf16"), (28, 4, 128, 128, False, "f32"), (3, 3, 64, 16, True, "none"),
    (10, 2, 128, 64, False, "q"), (8, 1, 128, 128, True, "bf16"), (4, 4, 128, 48, True, "f32"), (4, 4, 64, 48, False, "bf16")])
@pytest.mark.parametrize("e4m3", [False, True])
def test_rows_match_float64(lens, new, hq, hkv, d, rot, inter, weights, e4m3):
    c = Call(lens, new, hq, hkv, d, rot, e4m3=e4m3, interleaved=inter, pad=3, seed=len(lens) + d, weights=weights)
    c.run()
    c.check()


@pytest.mark.parametrize("e4m3,packed", [(False, False), (True, True)])
def test_many_sequences_single_tokens_and_positions(e4m3, packed):
    lens = [(13 * b) % 90 + 1 for b in range(150)]
    for offsets in (True, False):
        c = Call(lens, [1] * 150, 12, 2, 128, 128, e4m3=e4m3, packed=packed, seed=4, positions=offsets, offsets=offsets)
        c.run()
        c.check()


def test_large_prompts_share_workgroups():
    c = Call([4500, 600], [4500, 599], 2, 1, 64, 64, seed=15, pad=3)
    c.run()
    c.check()


def test_without_rotation_and_without_queries():
    for e4m3 in (False, True):
        c = Call([40, 7], [30, 7], 8, 2, 128, 128, e4m3=e4m3, scales=False, seed=7, with_q=False,
                 inv_freq=torch.zeros(0))
        c.run()
        c.check()


@pytest.mark.parametrize("gain,eps", [(1e-4, 1e-6), (1e-4, 1e-12), (1e6, 1e-5), (1.0, 0.0), (3e-3, 1.0)])
def test_sizes_and_eps(gain, eps):
    c = Call([20, 50], [20, 9], 6, 2, 128, 64, seed=16, gain=gain, eps=eps)
    c.run()
    c.check()


def test_heads_of_zeros_and_of_nan():
    """A head of zeros stays zeros; one with a NaN or an infinite element spoils itself alone."""
    c = Call([20], [20], 6, 2, 128, 128, seed=17)
    c.gpu[0][3, 2], c.gpu[1][4, 1] = 0, 0
    c.gpu[0][5, 1, 9], c.gpu[1][6, 0, 0] = float("nan"), float("inf")
    want = Call([20], [20], 6, 2, 128, 128, seed=17)
    for x in (c, want):
        x.run()
    torch.cuda.synchronize()
    assert not c.out[3, 2].any() and not c.kv_gpu[0][int(c.cache.table[0, 0]), 1, 4].any()
    assert bool(c.out[5, 1].isnan().all())
    changed = [(3, 2), (5, 1)]
    keep = torch.ones((20, 6), dtype=torch.bool)
    for i in changed:
        keep[i] = False
    assert torch.equal(c.out[keep.cuda()], want.out[keep.cuda()])
    k = [x.kv_gpu[0].clone() for x in (c, want)]
    for t, h in ((4, 1), (6, 0)):
        for x in k:
            x[int(c.cache.table[0, 0]), h, t] = 0
    assert torch.equal(k[0].view(torch.int16), k[1].view(torch.int16))


def test_runs_without_room_are_skipped():
    c = Call([20, 3, 33, 10], [4, 5, 2, 10], 8, 2, 64, 64, seed=8, width=3)
    c.lens[2] = 49   # three pages hold 48
    c.seq_lens[2] = 49
    c.run()
    c.check()


def test_in_place():
    c = Call([30, 9], [12, 9], 8, 2, 128, 128, packed=False, seed=9)
    c.q = c.q.clone()
    c.out = c.gpu[0]
    c.run()
    c.check()


def test_a_norm_of_ones_differs_from_none():
    """Without a norm the plain append's bits are what they were: the two entries stand beside each other."""
    c, plain = (k([40, 17], [9, 17], 12, 2, 128, 128, seed=11) for k in (Call, RopeCall))
    c.run()
    plain.run()
    c.check()
    plain.check()


def test_refusals():
    c = Call([20, 30], [2, 3], 8, 2, 64, 64, seed=13)
    q, k, v = c.gpu
    f = c.inv_freq.cuda()
    w = c.weights[0].cuda()

    def call(error, match, **kw):
        a = dict(q=q, k=k, v=v, out=c.out, qw=w, kw=None, eps=1e-6, f=f, off=c.offsets, pos=None)
        a.update(kw)
        with pytest.raises(error, match=match):
            T().delta_norm_rope_append(c.shape, c.kv, a["q"], a["k"], a["v"], a["out"], a["qw"], a["kw"], a["eps"],
                                       a["f"], row_offsets=a["off"], positions=a["pos"])
    call(ValueError, "^k: expected shape", k=k[:, :1])
    call(ValueError, "^v: 4 rows", v=v[:4])
    call(ValueError, "^q: 4 rows", q=q[:4])
    call(ValueError, "come together", q=None)
    call(ValueError, "^q_weight: expected shape", qw=w[:32].contiguous())
    call(ValueError, "^q_weight: expected torch.float32", kw=w.float())
    call(ValueError, "^k_weight: expected torch.bfloat16", kw=w.double())
    call(ValueError, "^k_weight: must be a GPU", kw=w.cpu())
    call(TypeError, "^q_weight: expected a torch.Tensor", qw=1.0)
    call(ValueError, "^row_offsets: expected shape", off=c.offsets[:2])
    call(ValueError, "^positions: nothing", f=None, pos=torch.zeros(5, dtype=torch.int32, device="cuda"))
    err = D().DeltaError
    call(err, "invalid argument", eps=-1.0)
    call(err, "invalid argument", eps=float("nan"))
    call(err, "invalid argument", eps=float("inf"))
    call(err, "invalid argument", qw=torch.zeros(65, dtype=torch.bfloat16, device="cuda")[1:])
    call(err, "invalid argument", f=f[:3].contiguous())
    call(err, "invalid argument", off=None)
    torch.cuda.synchronize()
    c.lens, c.new = [20, 30], [0, 0]
    c.check()   # nothing was written
    assert D()._lib.delta_norm_rope_append(ctypes.byref(c.shape), ctypes.byref(c.kv), None, None, 5,
                                           c.offsets.data_ptr(), None, 0, k.data_ptr(), 768, v.data_ptr(), 768,
                                           None, None) == -1
