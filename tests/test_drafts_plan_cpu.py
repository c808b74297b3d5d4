"""The cut of delta_tree_attn: every block of every tile is taken once, by groups that exist, the parts of a tile are
where the join looks for them, and no workgroup leaves more than its two."""
import random

import pytest

import draft_plan as P

HEADS = [(32, 8), (28, 4), (40, 8), (12, 2), (10, 2), (8, 1), (5, 5), (64, 64), (48, 6)]


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return P.build(str(tmp_path_factory.mktemp("plan")))


def draw(rng):
    hq, hkv = rng.choice(HEADS)
    batch = rng.choice([1, 1, 2, 3, 8, 16, 33, 64, 200, 256])
    longest = rng.choice([1, 2, 4, 7, 8, 9, 16, 24, 40, 64, 100, 300, 512])
    bound = int(2 ** rng.uniform(0, 17))
    new = [rng.choice([0, 1, longest, rng.randint(0, longest)]) for _ in range(batch)]
    lens = [rng.choice([bound, rng.randint(0, bound), 0]) for _ in range(batch)]
    rows = max(sum(new) + rng.choice([0, 5]), longest)
    return (batch, hq, hkv, bound, rows, longest), lens, new


def test_every_block_is_taken_once(exe):
    rng = random.Random(4)
    draws = [draw(rng) for _ in range(1500)]
    plans = P.ask(exe, [d[0] for d in draws])
    modes = {"few": 0, "pieces": 0, "equal": 0, "alone": 0}
    for (call, lens, new), plan in zip(draws, plans):
        batch, hq, hkv, bound, rows, longest = call
        assert plan.rows in (32, 256) and plan.tiles <= batch * -(-longest * hq // hkv // plan.rows) + batch
        modes["few"] += plan.rows == 32
        if plan.workgroups == 0:
            modes["alone"] += 1
            assert bound <= 768 or batch > 256
            tiles = sum(-(-n * (hq // hkv) // plan.rows) for n in new)
            assert tiles <= plan.tiles   # (a grid of so many)
            continue
        assert plan.workgroups % hkv == 0 and plan.workgroups // hkv <= 1023
        modes["pieces" if plan.pieces else "equal"] += 1
        for kv8 in (False, True):
            taken, said = P.shares(plan, hkv, hq // hkv, lens, new, kv8)
            blocks, places = {}, {}
            for g, b, t, lo, hi, n in taken:
                assert 0 <= g < plan.workgroups // hkv
                blocks.setdefault((b, t), []).append((lo, hi, g, n))
            for key, parts in blocks.items():
                parts.sort()
                assert parts[0][0] == 0 and parts[-1][1] == parts[0][3]
                assert all(x[1] == y[0] for x, y in zip(parts, parts[1:]))
                first, count = said[key]
                assert [p[2] for p in parts] == list(range(first, first + count))   # where the join looks for them
                if count > 1:
                    for i, p in enumerate(parts):
                        place = (p[2], i == 0)
                        assert place not in places, "two parts in one place"
                        places[place] = key
            want = {(b, t) for b, n in enumerate(new) for t in range(-(-n * (hq // hkv) // plan.rows))}
            assert set(blocks) == want
    assert all(modes.values()), modes


def test_calls_with_little_to_walk_take_small_tiles(exe):
    cases = [((1, 28, 4, 8192, 16, 16), 32), ((1, 28, 4, 32768, 16, 16), 256), ((16, 32, 8, 16384, 1024, 64), 256),
             ((16, 32, 8, 16384, 128, 8), 32), ((300, 32, 8, 16384, 300 * 64, 64), 256)]
    for (call, rows), plan in zip(cases, P.ask(exe, [c for c, _ in cases])):
        assert plan.rows == rows
