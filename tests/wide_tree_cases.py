"""Calls of delta_tree_attn that its plan sends to tiles of 256 rows (a host test holds that they still go
there), and all their rows in float64."""
from __future__ import annotations

import random

import torch

# tokens held, rows of the runs, query heads, KV heads, bound of the lengths (None: the longest)
WIDE = [
    # pieces of one tile each: up to 128 rows a KV head, more, and both in one call; empty runs and sequences
    ((1500, 700, 90, 1100, 0), (25, 16, 25, 0, 0), 40, 8, 8192),
    ((1500, 900, 33, 1100, 64), (64, 40, 33, 0, 17), 32, 8, None),
    ((1200, 1100), (120, 60), 32, 8, None),
    ((2000, 300), (9, 9), 64, 8, 131072),
    # runs of several tiles, whose borders are inside a token's heads (5, 6 and 7 a group), the last of few rows
    ((1400, 1000, 90), (200, 77, 12), 48, 8, None),
    ((1100, 40, 777), (300, 40, 1), 28, 4, None),
    ((4000,), (512,), 10, 2, None),
    # one and eight query heads a group, the longest runs
    ((900, 530), (512, 300), 4, 4, 60000),
    ((2000,), (512,), 8, 1, None),
    # long parts of one tile: a workgroup's ring goes round many times
    ((5000,), (100,), 32, 8, None),
    ((9000, 500, 70), (60, 30, 2), 14, 2, None),
    # equal shares: tiles that end and begin inside a workgroup, of every kind
    (tuple(800 + 10 * i for i in range(20)), (40, 70, 9, 33) * 5, 32, 8, None),
    (tuple((37 * i) % 900 + 70 for i in range(64)), tuple((11 * i) % 67 for i in range(64)), 16, 16, None),
    ((1000, 100, 0, 40, 700, 300) * 9, (33, 100, 0, 1, 65, 30) * 9, 20, 4, None),
    # a run longer than its sequence: its first rows' tokens are none
    ((40, 900, 3), (60, 100, 20), 32, 8, 40000),
    # short sequences, not shared
    ((700, 600, 500, 768, 90, 300), (60, 63, 20, 64, 64, 0), 32, 8, None),
    ((100,) * 12, (100,) * 12, 64, 8, None),
    # more sequences than are shared out, long and short, most of them without rows
    ((1500, 17, 1200, 0) * 66, (70, 0, 9, 0) + (0, 3, 0, 0) * 65, 16, 2, None),
]

# ... with values of tokens that a row does not see: (tokens, rows), the token; 32/8 heads beside a short run
HIDDEN = [((1000, 30), 990), ((1000, 33), 968), ((900, 400), 520), ((1300, 120), 1180), ((1301, 20), 1299),
          ((400, 400), 0), ((1100, 70), 1040)]


def hidden_call(case):
    (held, new), _ = case
    return (held, 20), (new, 3), 32, 8, 131072


# ... captured and replayed (in pieces and in equal shares), with scores that one token decides, with masks of any
# bits, and with rows that see nothing
REPLAYS = [((2000, 77, 900), (20, 64, 33), 32, 8, None), (tuple(900 + 5 * i for i in range(24)), (40, 70, 9, 33) * 6, 32, 8, None)]
SHARP = ((900, 1300), (90, 200), 32, 8, None)
BITS = ((1000, 300, 90, 33), (70, 100, 40, 33), 32, 8, None)
NOTHING = ((1000, 90, 64, 0), (100, 90, 64, 5), 32, 8, None)

# Calls that take tiles of 32 rows, whatever the number of heads (query heads a group, KV heads)
SMALL_TILES = [((3, 8, 20, 41), (3, 4, 4, 2)), ((150, 700, 64, 1), (4, 2, 3, 1)), ((40, 300, 90), (40, 33, 64)),
               ((2600, 1900), (4, 3)), ((9000,), (4,))]
SMALL_HEADS = [(1, 4), (4, 2), (7, 1)]

# ... of one workgroup that walks more pages than it looks up at a time: more sequences than are shared out
PAGES = ((16500, 35000, 17000), (70, 20, 9))


def pages_call():
    lens, new = PAGES
    return lens + (1,) * 260, new + (0,) * 259 + (1,), 8, 1, None


# ... whose pages stand at both ends of a cache of more than 2^32 elements: tokens, rows, query heads, KV heads
FAR = ((75, 45), 32, 8, 131072)


def drawn(count):
    """Calls of any such kind."""
    rng, out = random.Random(11), []
    while len(out) < count:
        hkv = rng.choice([1, 2, 3, 4, 8, 16])
        hq = hkv * rng.choice([1, 2, 3, 4, 5, 6, 7, 8])
        batch = rng.choice([1, 2, 3, 5, 9, 20, 40])
        longest = rng.choice([12, 20, 33, 64, 65, 100, 129, 300, 512])
        bound = int(2 ** rng.uniform(5, 11.5))
        lens = [rng.choice([bound, rng.randint(0, bound), rng.randint(0, bound)]) for _ in range(batch)]
        new = [rng.choice([0, 1, longest, rng.randint(0, longest), rng.randint(0, longest)]) for _ in range(batch)]
        if longest * hq // hkv <= 32 or sum(new) < longest or sum(s * n for s, n in zip(lens, new)) * hq > 12e6:
            continue
        new[0] = longest
        bound = rng.choice([131072, max(lens) or 1, 5000])
        tiles = sum(-(-n * hq // hkv // 32) for n in new)
        if tiles * (bound // 128 + 1) > 8 * (256 // hkv):   # (more than a call of small tiles has to walk)
            out.append((tuple(lens), tuple(new), hq, hkv, bound))
    return out


def plan_call(case, pad=0, more=0):
    """What the plan goes by: batch, heads, bound, rows, longest run."""
    lens, new, hq, hkv, bound = case
    return len(lens), hq, hkv, bound or max(lens), sum(new) + pad, max(new) + more


def attend_runs(call, k_of=None, v_of=None, p_round=None):
    """float64 outputs [rows, hq, d] of all rows of the runs of a test_gpu_tree_attn.Call, and how far a
    device result may be off: the bound of cache_cases.attend, row by row, with the values' largest of all
    the sequence's.  k_of, v_of: a sequence's keys and values instead of the cache's."""
    c, outs, tols = call, [], []
    p_round = P_ROUND if p_round is None else p_round
    hkv, d = c.cache.hkv, c.q.shape[2]
    G, row = c.hq // hkv, 0
    for b, (s, n) in enumerate(zip(c.lens, c.new)):
        sees = torch.zeros((n, s), dtype=torch.bool)
        for j in range(n):
            sees[j, c.tokens(b, j)] = True
        out = torch.zeros((n, c.hq, d), dtype=torch.float64)
        tol = torch.zeros_like(out)
        if n and s:
            k = k_of(b) if k_of else c.cache.tokens(0, b, range(s))
            v = v_of(b) if v_of else c.cache.tokens(1, b, range(s))
            some = sees.any(1).repeat_interleave(G)[:, None]
            hidden = ~sees.repeat_interleave(G, 0)
            for h in range(hkv):
                q = c.q[row:row + n, h * G:(h + 1) * G].double().reshape(n * G, d)
                x = (q @ k[:, h].t().contiguous() * c.scale).masked_fill(hidden, float("-inf"))
                e = (q.abs() @ k[:, h].abs().t().contiguous() * c.scale).masked_fill(hidden, 0).amax(1, keepdim=True)
                p = torch.where(some, torch.softmax(x, -1), 0.0)
                o = p @ v[:, h].contiguous()
                t = p_round * (p @ v[:, h].abs().contiguous()) + o.abs() * 2.0 ** -8
                t += 2 * (e * (d + 4) * 2.0 ** -24 + 2.0 ** -22 + s * 2.0 ** -24) * v[:, h].abs().max()
                out[:, h * G:(h + 1) * G] = o.view(n, G, d)
                tol[:, h * G:(h + 1) * G] = torch.where(some, t, 0.0).view(n, G, d)
        outs.append(out)
        tols.append(tol)
        row += n
    return torch.cat(outs), torch.cat(tols)


P_ROUND = 2.0 ** -8   # probabilities are rounded to bf16 before they meet the values
