"""tests/test_gpu_tree_wide.py tests delta_tree_attn in tiles of 256 rows: its calls have to reach them, in every
way that such a call is cut, whatever becomes of the rule."""
import shutil

import pytest

import draft_plan as P
import wide_tree_cases as C

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return P.build(str(tmp_path_factory.mktemp("plan")))


def mode(plan):
    return "alone" if not plan.workgroups else "pieces" if plan.pieces else "equal"


def tiles_of(case):
    """Rows of every tile of 256."""
    lens, new, hq, hkv, _ = case
    rows = [n * (hq // hkv) for n in new]
    return [min(256, r - t) for r in rows for t in range(0, r, 256)]


def test_the_cases_take_tiles_of_256_rows_in_every_way(exe):
    met = set()
    for case, plan in zip(C.WIDE, P.ask(exe, [C.plan_call(c, pad=3) for c in C.WIDE])):
        assert plan.rows == 256, case
        met |= {(mode(plan), rows > 128) for rows in tiles_of(case)}
    assert met == {(m, wide) for m in ("alone", "pieces", "equal") for wide in (False, True)}


def test_workgroups_take_several_tiles_and_tiles_several_workgroups(exe):
    """Equal shares: a workgroup with parts of three tiles and more, a tile in three and more parts, of both kinds."""
    most, parts = 0, {False: 0, True: 0}
    for case, plan in zip(C.WIDE, P.ask(exe, [C.plan_call(c, pad=3) for c in C.WIDE])):
        if not plan.workgroups:
            continue
        lens, new, hq, hkv, _ = case
        for kv8 in (False, True):
            taken, said = P.shares(plan, hkv, hq // hkv, lens, new, kv8)
            if not plan.pieces:
                groups = [t[0] for t in taken]
                most = max(most, max(groups.count(g) for g in set(groups)))
            for (b, t), (_, count) in said.items():
                wide = min(256, new[b] * (hq // hkv) - 256 * t) > 128
                parts[wide] = max(parts[wide], count)
    assert most >= 3 and min(parts.values()) >= 3


def test_the_other_cases_too(exe):
    cases = [C.plan_call(C.hidden_call(h)) for h in C.HIDDEN] + [C.plan_call(c, pad=3) for c in C.drawn(30)]
    cases += [*map(C.plan_call, C.REPLAYS), C.plan_call(C.SHARP, pad=200, more=2), C.plan_call(C.BITS), C.plan_call(C.NOTHING)]
    (held, n), hq, hkv, bound = C.FAR
    cases.append((1, hq, hkv, bound, n, n))
    for call, plan in zip(cases, P.ask(exe, cases)):
        assert plan.rows == 256, call
    plan = P.ask(exe, [C.plan_call(C.pages_call())])[0]
    assert plan.rows == 256 and not plan.workgroups    # a workgroup walks its tile's whole sequence


def test_the_cases_of_small_tiles_take_them(exe):
    calls = [C.plan_call((lens, new, G * hkv, hkv, None)) for lens, new in C.SMALL_TILES for G, hkv in C.SMALL_HEADS]
    assert {p.rows for p in P.ask(exe, calls)} == {32}


def test_shapes_of_the_cases_are_taken():
    from paper_2510_09883_amd import delta as D
    from paper_2510_09883_amd import drafts as T
    for lens, new, hq, hkv, bound in (*C.WIDE, *C.drawn(30), C.pages_call()):
        bound = bound or max(lens)
        for d in (64, 128):
            shape = D.make_shape(len(lens), hq, hkv, d, -(-bound // 16), bound)
            assert T.delta_tree_workspace_bytes(shape, sum(new) + 3, max(new)) > 0
