"""How the library cuts calls of delta_tree_attn: its plan, asked of the rule itself (plan_tree of
csrc/drafts_api.cpp, compiled for the host), and a model of the shares that the kernel forms from it."""
from __future__ import annotations

import os
import subprocess
from collections import namedtuple

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2510_09883_amd", "csrc")

# rows of a tile, most tiles, workgroups of a shared call (0: not shared), pieces or equal shares
Plan = namedtuple("Plan", "rows tiles workgroups pieces tile_units least_units")

MAIN = r"""
#include <cstdio>
#include "%s/drafts.h"
namespace delta {
hipError_t launch_rope_append(int, bool, const RopeAppendArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_norm_rope_append(int, bool, const RopeAppendArgs&, const HeadNorm&, hipStream_t) { return hipSuccess; }
hipError_t launch_extend(const ExtendPlan&, int, bool, const ExtendArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_tree_layout(const TreeLayoutArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_tree_attn(const TreePlan&, int, bool, const ExtendArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_verify(const VerifyArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_compact(const CompactArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_compact_lens(const CompactArgs&, hipStream_t) { return hipSuccess; }
}
int main() {
  int b, hq, hkv, len, rows, longest;
  while (scanf("%%d %%d %%d %%d %%d %%d", &b, &hq, &hkv, &len, &rows, &longest) == 6) {
    const delta_shape_t s{b, hq, hkv, 128, 16, (int)(((long)len + 15) / 16), len, 0.f};
    const delta::TreePlan p = delta::plan_tree(&s, rows, longest);
    printf("%%d %%d %%d %%d %%d %%d\n", p.rows, p.tiles, p.workgroups, (int)p.pieces, delta::kTileUnits, delta::kLeastUnits);
  }
}
"""


def build(folder):
    """The program, compiled into `folder`."""
    src, exe = os.path.join(folder, "plan.cpp"), os.path.join(folder, "plan")
    with open(src, "w") as f:
        f.write(MAIN % CSRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I",
                    os.path.join(ROOT, "include"), src, os.path.join(CSRC, "drafts_api.cpp"),
                    os.path.join(CSRC, "extend_api.cpp"), "-o", exe], check=True)
    return exe


def ask(exe, calls):
    """Plans of calls (batch, n_q_heads, n_kv_heads, max_seq_len, n_rows, max_new)."""
    text = "".join("%d %d %d %d %d %d\n" % (*c[:4], min(c[4], c[0] * c[5]), c[5]) for c in calls)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
    return [Plan(*map(int, line.split())) for line in out.splitlines()]


def form_of(plan, kv8, rows):
    """Keys and units of a block for a tile of so many rows (form_of of csrc/tree_attn_kernel.hip)."""
    if plan.rows == 32:
        return 128, 4 if kv8 else 8
    if rows <= 128:
        return (128, 6) if kv8 else (64, 4)
    return 64, 6


def shares(plan, heads, group, lens, new, kv8):
    """What every group of workgroups takes: (group, sequence, tile, first block, end block, blocks of the tile), and
    the groups that each tile's parts are said to be in: {(sequence, tile): (first group, count)}."""
    W, R = plan.workgroups // heads, plan.rows
    tiles = []   # (sequence, tile, blocks, units of a block)
    for b, (s, n) in enumerate(zip(lens, new)):
        rows = n * group
        for t in range(-(-rows // R)):
            keys, units = form_of(plan, kv8, min(R, rows - t * R))
            tiles.append((b, t, max(1, -(-s // keys)), units))
    total = sum(x[2] * x[3] for x in tiles)
    taken, said = [], {}
    if plan.pieces:
        chunk = max(plan.least_units, -(-total // max(1, W - len(tiles))))
        g = 0
        for b, t, blocks, units in tiles:
            per = -(-chunk // units)
            count = -(-blocks // per)
            said[b, t] = (g, count)
            for i in range(count):
                taken.append((g, b, t, i * per, min(blocks, (i + 1) * per), blocks))
                g += 1
        assert g <= W, "pieces without a workgroup"
        return taken, said
    total += plan.tile_units * len(tiles)
    chunk = max(plan.least_units, -(-total // W))
    start = 0
    for b, t, blocks, units in tiles:
        end = start + plan.tile_units + blocks * units
        for g in range(start // chunk, (end - 1) // chunk + 1):
            assert g < W, "units without a workgroup"

            def block_from(unit):
                return min(blocks, -(-max(0, unit - plan.tile_units) // units))
            lo = block_from(max(g * chunk, start) - start)
            hi = block_from(min((g + 1) * chunk, end if (g + 1) * chunk > end else (g + 1) * chunk) - start)
            if lo < hi:
                taken.append((g, b, t, lo, hi, blocks))
                if lo == 0:
                    said[b, t] = (g, (start + plan.tile_units + (blocks - 1) * units) // chunk - g + 1)
        start = end
    return taken, said
