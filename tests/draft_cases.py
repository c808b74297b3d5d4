"""Trees of drafted tokens for the tests: parents, what rows see, and the verification in exact arithmetic."""
from __future__ import annotations

from fractions import Fraction

import torch


def tree(n, kind, seed=0):
    """Parents of n rows: a chain, a star (all continue the first), a bush (random earlier rows), pairs
    (binary tree), or roots (none continues another)."""
    g = torch.Generator().manual_seed(seed)
    if n == 0:
        return []
    if kind == "chain":
        return [j - 1 for j in range(n)]
    if kind == "star":
        return [-1] + [0] * (n - 1)
    if kind == "pairs":
        return [-1] + [(j - 1) // 2 for j in range(1, n)]
    if kind == "roots":
        return [-1] * n
    return [-1] + [int(torch.randint(max(0, j - 6), j, (1,), generator=g)) for j in range(1, n)]


def sees_of(parents):
    """Depths, and for every row the set of places that it sees."""
    depths, sets = [], []
    for j, p in enumerate(parents):
        ok = 0 <= p < j
        depths.append(depths[p] + 1 if ok else 0)
        sets.append((sets[p] if ok else frozenset()) | {j})
    return depths, sets


def mask_words(sets, words):
    """int32 [rows, words] of sets of places."""
    out = torch.zeros((len(sets), words), dtype=torch.int64)
    for r, places in enumerate(sets):
        for i in places:
            out[r, i // 32] |= 1 << (i % 32)
    return torch.where(out >= 2 ** 31, out - 2 ** 32, out).int()


def offsets_of(new):
    return torch.tensor([0] + torch.tensor(new, dtype=torch.long).cumsum(0).tolist(), dtype=torch.int32)


def _fractions(row):
    """A row of probabilities as exact numbers; NaN and negative ones count as 0."""
    return [Fraction(x) if x == x and x > 0 else Fraction(0) for x in row.double().tolist()]


def verified(target, draft, tokens, parents, uniform):
    """One run: (places of the accepted rows, the next token), from the definition in exact arithmetic, one
    row of probabilities at a time."""
    n, vocab = target.shape
    if n == 0:
        return [], -1
    path = [0]
    while True:
        cur = path[-1]
        p = _fractions(target[cur])
        r, mass = list(p), Fraction(1)
        q = _fractions(draft[cur]) if draft is not None else None
        step = None
        for j in range(cur + 1, n):
            if parents[j] != cur:
                continue
            x = tokens[j]
            have = r[x] if 0 <= x < vocab else Fraction(0)
            chance = (q[x] if 0 <= x < vocab else Fraction(0)) if draft is not None else 1
            if Fraction(float(uniform[j])) * chance * mass < have:
                step = j
                break
            if draft is None:
                if 0 <= x < vocab:
                    r[x] = Fraction(0)
                mass = max(mass - have, 0)
            else:
                r = [max(a - mass * b, 0) for a, b in zip(r, q)]
                mass = sum(r)
        if step is None:
            break
        path.append(step)
    if sum(r) == 0:
        r = p
    total = sum(r)
    if total == 0:
        return path, -1
    goal, cum, last = Fraction(float(uniform[0])) * total, Fraction(0), -1
    for v, x in enumerate(r):
        if x > 0:
            last = v
        cum += x
        if cum > goal:
            return path, v
    return path, last
