"""The cut of delta_extend_attn calls (plan_extend) on the host: which kernel, how many tiles and pieces."""
import ctypes
import random
import shutil

import pytest

import extend_plan as P
import many_row_cases as C
from paper_2510_09883_amd import delta as D

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return P.build(str(tmp_path_factory.mktemp("plan")))


LONGEST = 2 ** 31 - 512   # the longest bound that delta_extend_attn takes


def _calls():
    rng = random.Random(5)
    for held in (1, 255, 256, 257, 4096, 131072, 2 ** 30, 2 ** 30 + 1, 2 ** 30 + 300, 1200000000, LONGEST):
        for batch, n_rows, longest in ((1, 1, 1), (1, 4, 4), (1, 4000, 4000), (64, 4000, 400), (300, 300, 1)):
            yield batch, 8, 2, 128, held, n_rows, longest
    for _ in range(300):
        G, hkv = rng.randint(1, 8), rng.randint(1, 8)
        batch = int(2 ** rng.uniform(0, 12))
        longest = int(2 ** rng.uniform(0, 12))
        n_rows = max(longest, int(batch * longest * rng.uniform(0.1, 1.0)))
        yield batch, G * hkv, hkv, rng.choice([64, 128]), int(2 ** rng.uniform(0, 30.9)), n_rows, longest


def test_pieces_cover_every_length(exe):
    """Pieces of whole blocks that cover the host's bound, at most 32, none of them behind it."""
    calls = list(_calls())
    for c, p in zip(calls, P.ask(exe, calls)):
        assert 1 <= p.n_split <= 32, (c, p)
        assert p.split_keys % 256 == 0 and p.n_split * p.split_keys >= c[4], (c, p)
        assert (p.n_split - 1) * p.split_keys < c[4], (c, p)
        assert p.n_split == 1 or p.n_split * min(c[5], c[0] * c[6]) * c[1] <= 1 << 17, (c, p)


def test_bounds_past_the_kernels_arithmetic_are_refused():
    """The kernels round key indices up to whole blocks in 32 bits."""
    fake = ctypes.c_void_p(0x1000)
    for held, rc in ((LONGEST, D.DELTA_ERR_INVALID_ARG), (LONGEST + 1, D.DELTA_ERR_UNSUPPORTED),
                     (2 ** 31 - 1, D.DELTA_ERR_UNSUPPORTED)):
        s = D.make_shape(1, 8, 2, 128, 1 << 27, held)
        kv = D.delta_kv_t(0x1000, 0x1000, 0x1000, 0x1000, 0)
        assert D._lib.delta_extend_attn(ctypes.byref(s), ctypes.byref(kv), 4, 4, fake, None, fake, fake, 1 << 40,
                                        None) == rc   # (null queries: refused after the bound)
        size = ctypes.c_size_t(0)
        taken = D._lib.delta_extend_workspace_bytes(ctypes.byref(s), 4, 4, ctypes.byref(size)) == D.DELTA_OK
        assert taken == (held <= LONGEST)


def test_the_cases_of_many_rows_go_to_that_kernel(exe):
    """tests/test_gpu_extend_many_rows.py tests the kernel of 256-row tiles: its calls have to reach it,
    with one piece of the keys and with several, whatever becomes of the rule."""
    cases = [C.plan_call(*c, d) for c in (*C.MANY_ROWS, C.HIDDEN) for d in (64, 128)]
    batch, held, new, hq, hkv = C.MOST_TILES
    cases += [(batch, hq, hkv, 64, held, batch * new, new), (2, 10, 2, 128, 1800, 1502, 1450)]
    plans = P.ask(exe, cases)
    assert [p.rows for p in plans] == [256] * len(cases), [c for c, p in zip(cases, plans) if p.rows != 256]
    assert {p.n_split > 1 for p in plans} == {False, True}
