"""The LDS of the rings of e4m3 blocks that tree attention loads (csrc/attend_lds.h, compiled for the host): every
wave reads and writes LDS of its own, inside the workgroup's, and every piece of a block is one wave's."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_09883_amd", "csrc")

MAIN = r"""
#include <cstdio>
#include "attend_lds.h"
using namespace delta;
template <int D> void list() {
  typedef RawRing<D, 8, 64> Raw;   // (extend_body<D, 8, 1, 2, true, true, true>)
  printf("%d 0 0 0 %d %d\n", D, Raw::kBegin, kBodyLds<D, 8, 1, 2, true, true>);
  for (int wave = 0; wave < 8; ++wave)
    for (int load = 0; load < Raw::kLoads; ++load)
      for (int stage = 0; stage < kRing; ++stage)
        if (Raw::has(wave, load)) printf("%d %d %d %d %d %d\n", D, wave, load, stage, Raw::at(wave, stage, load), 2048);
}
int main() { list<64>(); list<128>(); }
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_waves_of_an_e4m3_ring_stay_in_their_own_lds(tmp_path):
    src, exe = tmp_path / "lds.cpp", tmp_path / "lds"
    src.write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    lines = [tuple(map(int, x.split())) for x in out.splitlines()]
    for d in (64, 128):
        begin, size = next(x[4:] for x in lines if x[0] == d)
        taken = [x for x in lines if x[0] == d][1:]
        assert begin == 2 * 2 * 64 * d * 2                 # behind two buffers of K and V as bf16
        places = sorted(x[4] for x in taken)
        assert places[0] >= begin and places[-1] + 2048 <= size
        assert all(b - a >= 2048 for a, b in zip(places, places[1:]))
        # 64 pieces of 16 bytes a load: a block of K (and of V) in each stage, once
        for stage in range(4):
            assert sum(64 * 16 for x in taken if x[3] == stage) == 64 * d


def test_the_kernel_reads_by_that_layout():
    """Each of the ring's LDS reads and loads of e4m3 blocks goes by the layout's own guard and places."""
    text = open(os.path.join(CSRC, "attend_runs.h")).read()
    body = text[text.index("if constexpr (RING) {"):text.index("} else if (blk0 < blk1) {")]
    assert body.count("Raw::at(wave, stage, i)") == 2 and body.count("!Raw::has(wave, i)) break") == 1
    assert body.index("!Raw::has(wave, i)) break") < body.index("kr[i] =")
