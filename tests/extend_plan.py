"""How the library cuts calls of delta_extend_attn, asked of its own rule: plan_extend of
csrc/extend_api.cpp is compiled for the host with a program that prints its answers."""
from __future__ import annotations

import os
import subprocess
from collections import namedtuple

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2510_09883_amd", "csrc")

# rows of a tile (32: the few-row kernel, 256: the many-row kernel), tiles of the grid, pieces of the
# keys and keys of a piece
Plan = namedtuple("Plan", "rows tiles n_split split_keys")

MAIN = r"""
#include <cstdio>
#include "%s/extend.h"
namespace delta {
hipError_t launch_rope_append(int, bool, const RopeAppendArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_extend(const ExtendPlan&, int, bool, const ExtendArgs&, hipStream_t) { return hipSuccess; }
}
int main() {
  int b, hq, hkv, d, len, rows, longest;
  while (scanf("%%d %%d %%d %%d %%d %%d %%d", &b, &hq, &hkv, &d, &len, &rows, &longest) == 7) {
    const delta_shape_t s{b, hq, hkv, d, 16, (int)(((long)len + 15) / 16), len, 0.f};
    const delta::ExtendPlan p = delta::plan_extend(&s, rows, longest);
    printf("%%d %%d %%d %%d\n", p.rows, p.tiles, p.n_split, p.split_keys);
  }
}
"""


def build(folder):
    """The program, compiled into `folder`."""
    src, exe = os.path.join(folder, "plan.cpp"), os.path.join(folder, "plan")
    with open(src, "w") as f:
        f.write(MAIN % CSRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
                    "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), src,
                    os.path.join(CSRC, "extend_api.cpp"), "-o", exe], check=True)
    return exe


def ask(exe, calls):
    """Plans of calls (batch, n_q_heads, n_kv_heads, head_dim, max_seq_len, n_rows, max_new), max_new at
    most n_rows."""
    # (rows that can belong to a run: what the entry point hands to the rule)
    text = "".join("%d %d %d %d %d %d %d\n" % (*c[:5], min(c[5], c[0] * c[6]), c[6]) for c in calls)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
    return [Plan(*map(int, line.split())) for line in out.splitlines()]
