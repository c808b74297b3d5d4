"""How many bits of the probabilities delta_tree_attn keeps: two bf16 terms in tiles of 32 rows of bf16 caches (at most
2^-8 of what the first leaves, 2^-8 of each), fp16 over e4m3 caches (half of a step is at most 2^-11 of a value).  Outputs
that are small beside the terms that they are summed from tell."""
import pytest

import wide_tree_cases as C
from cache_cases import worst
from test_gpu_tree_attn import Call

pytestmark = pytest.mark.gpu


def check(c, p_round):
    import torch
    torch.cuda.synchronize()
    want, tol = C.attend_runs(c, p_round=p_round)
    assert worst(c.out.cpu()[:want.shape[0]], want, tol) <= 1


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,hkv", C.SMALL_HEADS)
@pytest.mark.parametrize("lens,new", C.SMALL_TILES)
def test_two_terms_of_bf16_caches(lens, new, G, hkv, d):
    c = Call(list(lens), list(new), G * hkv, hkv, d, seed=sum(lens) + G)
    c.run()
    check(c, 2.0 ** -16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("k_gain", [1.0, 4.0])
@pytest.mark.parametrize("case", [((3, 8, 20, 41), (3, 4, 4, 2), 8, 2, None), ((150, 700, 64, 1), (4, 2, 3, 1), 8, 2, None),
                                  ((2600, 1900), (4, 3), 8, 2, None), ((40, 300, 90), (40, 33, 64), 8, 2, 131072),
                                  ((300, 900), (20, 31), 32, 8, 131072), *C.WIDE[:3], C.WIDE[11], C.WIDE[15], C.WIDE[17]])
def test_fp16_of_e4m3_caches(case, k_gain, d):
    lens, new, hq, hkv, bound = case
    c = Call(list(lens), list(new), hq, hkv, d, e4m3=True, seed=d + len(lens), bound=bound, k_gain=k_gain,
             width=-(-(bound or max(lens)) // 16))
    c.run()
    check(c, 2.0 ** -11)


@pytest.mark.parametrize("d", [64, 128])
def test_the_largest_and_smallest_e4m3_values(d):
    """Values of 448 and of 2^-9, all that e4m3 has in between, and scores far apart: fp16 holds them all."""
    import torch
    for case in (((90, 40), (9, 4), 8, 2, None), C.WIDE[1]):
        lens, new, hq, hkv, bound = case
        c = Call(list(lens), list(new), hq, hkv, d, e4m3=True, seed=9, bound=bound, sm_scale=0.4,
                 width=-(-(bound or max(lens)) // 16))
        bytes_of = lambda x: x.view(torch.uint8)   # noqa: E731
        v = c.cache.stored[1]
        g = torch.Generator().manual_seed(4)
        new_bytes = torch.randint(0, 256, v.shape, generator=g).to(torch.uint8)
        new_bytes[(new_bytes & 0x7F) == 0x7F] = 0x7E
        held = bytes_of(v) != 0x7F                 # (rows of no sequence hold NaN)
        bytes_of(v)[held] = new_bytes[held]
        scale = c.cache.v_scale.double()[:, None, None]
        c.cache.values[1] = v.double() * scale
        c.kv._tensors[1].view(torch.uint8).copy_(bytes_of(v).cuda())
        c.run()
        check(c, 2.0 ** -11)
