"""Paged caches of bf16 or e4m3 values for the tests, their float64 contents, and attention over
them in float64 with a bound on what fp32 sums and one bf16 rounding may be off."""
from __future__ import annotations

import math

import torch

PAGE = 16


class Cache:
    """Shuffled pages of `lens` tokens a sequence, `spare` pages more.  Rows past a sequence's end,
    pages that no sequence owns and page-table entries past its pages hold NaN and page 0."""

    def __init__(self, lens, hkv, d, e4m3=False, scales=True, seed=0, spare=2, width=None, device="cuda",
                 k_gain=1.0):
        g = torch.Generator().manual_seed(seed)
        pages = [-(-s // PAGE) for s in lens]
        self.lens, self.hkv, self.d, self.e4m3, self.device = list(lens), hkv, d, e4m3, device
        n = max(1, sum(pages) + spare)
        pool = torch.randperm(n, generator=g)
        self.width = width or max(1, max(pages))
        self.table = torch.zeros((len(lens), self.width), dtype=torch.int32)
        at = 0
        for b, m in enumerate(pages):
            self.table[b, :m] = pool[at:at + m].int()
            at += m
        self.k_scale = self.v_scale = None
        if e4m3 and scales:
            self.k_scale = 0.02 + 0.1 * torch.rand((hkv,), generator=g)
            self.v_scale = 0.02 + 0.1 * torch.rand((hkv,), generator=g)
        self.stored, self.values = [], []     # CPU: what the cache holds, and what it stands for
        for scale, gain in ((self.k_scale, k_gain), (self.v_scale, 1.0)):
            x = torch.randn((n, hkv, PAGE, d), generator=g, dtype=torch.float64) * gain
            s = torch.ones((hkv,)) if scale is None else scale
            x = (x / s.double()[:, None, None]).clamp(-448, 448).float()
            x = x.to(torch.float8_e4m3fn if e4m3 else torch.bfloat16)
            owned = torch.zeros((n, PAGE), dtype=torch.bool)
            for b, length in enumerate(lens):
                for t in range(0, length, PAGE):
                    owned[self.table[b, t // PAGE], :min(PAGE, length - t)] = True
            raw = x.view(torch.uint8 if e4m3 else torch.int16)
            raw[(~owned)[:, None, :].expand(n, hkv, PAGE)] = 0x7F if e4m3 else 0x7FC0
            self.stored.append(x)
            self.values.append(x.double() * s.double()[:, None, None])

    def tokens(self, which, b, tokens):
        """float64 [n, hkv, d] of keys (0) or values (1) of sequence b's tokens."""
        t = torch.as_tensor(tokens, dtype=torch.long)
        return self.values[which][self.table[b, t // PAGE].long(), :, t % PAGE]

    def on_gpu(self, D):
        dev = [x.to(self.device) for x in self.stored]
        table = self.table.to(self.device)
        lens = torch.tensor(self.lens, dtype=torch.int32, device=self.device)
        sc = {n: s.to(self.device) for n, s in (("k_scale", self.k_scale), ("v_scale", self.v_scale))
              if s is not None}
        return D.make_kv(dev[0], dev[1], table, lens, **sc)


def queries(rows, hq, d, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((rows, hq, d), generator=g).to(torch.bfloat16)


def attend(q, k, v, scale, p_round=0.0):
    """float64 output [hq, d] of one row's queries over k, v [n, hkv, d], and how far a device
    result may be off in each output.

    Bound.  A score is a sum of d products in fp32 (bf16 products are exact), then a product by the
    scale and a difference: off by at most (d + 4) 2^-24 sum|q k| scale =: e; a probability by the
    factor exp(+-e) and another 2^-22 for exp2 and the rescalings; sums over n terms by n 2^-24; a
    split into bf16 terms of probabilities loses nothing.  Weighted by the softmax, numerator and
    denominator together are off by at most 2 (e + 2^-22 + n 2^-24) max|v|.  One rounding to bf16
    adds 2^-8 of the result.  p_round: probabilities are rounded by at most that part of each
    before they meet the values, which adds p_round sum p |v|."""
    hq, hkv = q.shape[0], k.shape[1]
    G = hq // hkv
    out = torch.zeros((hq, q.shape[1]), dtype=torch.float64)
    tol = torch.zeros_like(out)
    n = k.shape[0]
    if n == 0:
        return out, tol
    qd = q.double()
    for h in range(hkv):
        rows = slice(h * G, (h + 1) * G)
        s = qd[rows] @ k[:, h].t().contiguous() * scale
        e = (qd[rows].abs() @ k[:, h].abs().t().contiguous() * scale).max() * (q.shape[1] + 4) * 2.0 ** -24
        out[rows] = torch.softmax(s, -1) @ v[:, h].contiguous()
        tol[rows] = p_round * (torch.softmax(s, -1) @ v[:, h].abs().contiguous())
        tol[rows] += 2 * (e + 2.0 ** -22 + n * 2.0 ** -24) * v[:, h].abs().max() + out[rows].abs() * 2.0 ** -8
    return out, tol


def default_scale(d):
    return 1.0 / math.sqrt(d)


def worst(got, want, tol):
    """How far `got` is off in units of the tolerance (above 1, or NaN: wrong)."""
    if want.numel() == 0:
        return 0.0
    r = (got.double().cpu() - want).abs() / tol.clamp(min=1e-30)
    r = torch.where((want == 0) & (got.double().cpu() == 0), torch.zeros_like(r), r)
    return float("nan") if bool(r.isnan().any()) else float(r.max())
