#!/usr/bin/env python3
"""Decode-step attention benchmark: the full layer stack vs the DELTA layer stack on one GPU.

One step = one decoding step of every layer's attention over a full-resident paged bf16 KV
cache (inputs already in HBM): all-full roles for the full stack; full, Delta (attention +
page scoring + page selection) and sparse layers for the DELTA stack (App. A, Alg. 1).
Each step is one call of delta_decode_step, captured in a HIP graph and replayed; when a step
touches less than ~1 GiB, several copies of the inputs are rotated so that the 256 MB
Infinity Cache cannot serve a step from the previous one.

Printed JSON line (rank 0, N = 1): value = DELTA-stack microseconds per step (lower is
better), with the full stack, the per-step median / p10 / p90, tokens/s, algorithmic HBM GB/s,
per-role layer times and their fractions of the 8 TB/s peak and of the read rate a plain
streaming kernel reaches on this GPU, the Delta-select overhead, the roofline of the dominant
kernel (per-launch time from HIP events around graph-captured launches of that role on the
launch stream) and the CPU oracle timed on this host.

With --sweep, one JSON line per point of a runtime sweep over the paper's settings instead.
"""
from __future__ import annotations

import argparse
import json
import math
import os
import sys
import time

import torch

ROOT = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, ROOT)

from paper_2510_09883_amd import configs, synth  # noqa: E402

METRIC = "decode attention µs/step + achieved HBM GB/s (% peak), full vs DELTA stack"
HBM_PEAK_GBPS = 8000.0
# The paper's own headline figures, for context only: they are whole-model results on its own
# hardware and are neither measured nor targeted here.
PAPER_CONTEXT = {
    "attended_tokens": "up to 4.25x fewer attended tokens than the sparse-attention methods the "
                       "paper compares with, at matching accuracy (abstract; Sec. 1)",
    "end_to_end_speedup": "up to 1.54x end-to-end decoding speed-up over full attention "
                          "(Sec. 5.3)",
    "hardware": "NVIDIA A100 SXM4 40 GB, one node of eight (Sec. 5)",
}
ROLE_NAME = {configs.ROLE_FULL: "full", configs.ROLE_DELTA: "delta", configs.ROLE_SPARSE: "sparse"}


def log(msg):
    print(f"[bench {time.strftime('%H:%M:%S')}] {msg}", file=sys.stderr, flush=True)


# ------------------------------------------------------------------------------------------
# algorithmic bytes (what the method itself must move; logits/partials are overhead)
# ------------------------------------------------------------------------------------------
def full_layer_bytes(w, lens):
    kv = sum(4 * w.n_kv_heads * w.head_dim * s for s in lens)
    qo = 4 * w.n_q_heads * w.head_dim * w.batch
    pt = sum(4 * ((s + 15) // 16) for s in lens)
    return kv + qo + pt


def sparse_layer_bytes(w, lens, sel_idx, sel_cnt):
    """sel_idx [B, K_u], sel_cnt [B] (host): tokens of the selected units, clipped at s_b."""
    U = w.unit_tokens
    toks = 0
    for b, s in enumerate(lens):
        for u in sel_idx[b, :sel_cnt[b]].tolist():
            toks += min(U, s - u * U)
    kv = 4 * w.n_kv_heads * w.head_dim * toks
    qo = 4 * w.n_q_heads * w.head_dim * w.batch
    idx = 4 * w.budget_units * w.batch
    return kv + qo + idx


# ------------------------------------------------------------------------------------------
def build_sets(w, n_sets):
    log(f"generating inputs: {w.describe()}, {n_sets} rotating copies")
    base = synth.make_inputs(w, "cuda", poison_tail=False)
    sets = [base]
    for _ in range(1, n_sets):
        sets.append(synth.DecodeInputs(
            w, [k.clone() for k in base.k_cache], [v.clone() for v in base.v_cache],
            [q.clone() for q in base.q], base.page_table, base.seq_lens, base.seq_lens_host,
            base.max_pages_per_seq, base.n_phys_pages))
    torch.cuda.synchronize()
    return sets


class Stack:
    """Per-input-set step arguments and a captured graph for one role list."""

    def __init__(self, D, w, sets, roles, shape, sel, ws):
        self.D, self.roles, self.sets = D, roles, sets
        n_delta = max(1, sum(r == configs.ROLE_DELTA for r in roles))
        self.sel_idx = torch.zeros((n_delta, w.batch, w.budget_units), dtype=torch.int32, device="cuda")
        self.sel_cnt = torch.zeros((n_delta, w.batch), dtype=torch.int32, device="cuda")
        self.sel_phys = torch.zeros((n_delta, w.batch, w.budget_units), dtype=torch.int32, device="cuda")
        self.outs, self.args = [], []
        n = len(roles)
        for inp in sets:
            outs = [torch.empty_like(q) for q in inp.q[:n]]
            kvs = [D.make_kv(inp.k_cache[i], inp.v_cache[i], inp.page_table, inp.seq_lens)
                   for i in range(n)]
            self.outs.append(outs)
            self.args.append(D.StepArgs(shape, roles, kvs, inp.q[:n], outs, sel, self.sel_idx,
                                        self.sel_cnt, ws))
        self.graphs = []

    def eager(self, k):
        self.D.delta_decode_step(self.args[k % len(self.args)])

    def capture(self):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for a in self.args:
                self.D.delta_decode_step(a)
        torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        for a in self.args:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                self.D.delta_decode_step(a)
            self.graphs.append(g)
        torch.cuda.synchronize()

    def replay(self, k):
        self.graphs[k % len(self.graphs)].replay()


def time_steps(stack, steps, warmup):
    for k in range(warmup):
        stack.replay(k)
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    e0.record()
    for k in range(steps):
        stack.replay(k)
    e1.record()
    torch.cuda.synchronize()
    return e0.elapsed_time(e1) / steps   # ms per step


def step_distribution(stack, steps):
    """Per-step times (us) from HIP events between consecutive replays: median, p10, p90."""
    import numpy as np
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(steps + 1)]
    torch.cuda.synchronize()
    ev[0].record()
    for k in range(steps):
        stack.replay(k)
        ev[k + 1].record()
    torch.cuda.synchronize()
    t = np.array([ev[k].elapsed_time(ev[k + 1]) * 1e3 for k in range(steps)])
    return {"median": round(float(np.median(t)), 2), "p10": round(float(np.percentile(t, 10)), 2),
            "p90": round(float(np.percentile(t, 90)), 2)}


def read_ceiling(D):
    """The best streaming-read rate of the probe kernel (include/delta_probe.h) over a 4 GiB
    buffer, over a few launch shapes, each timed over 8 launches after 2 untimed ones: the
    read bandwidth this GPU delivers to a plain streaming kernel, beside the data-sheet peak."""
    nbytes = 4 << 30
    buf = torch.ones(nbytes // 4, dtype=torch.int32, device="cuda")
    best = (0.0, None)
    for wgs in (256, 512, 1024, 2048):
        for unroll in (2, 4, 8):
            sink = torch.zeros(wgs, dtype=torch.int32, device="cuda")
            for _ in range(2):
                D.delta_hbm_read_probe(buf, sink, wgs, unroll)
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
            for _ in range(8):
                D.delta_hbm_read_probe(buf, sink, wgs, unroll)
            e1.record()
            torch.cuda.synchronize()
            gbps = nbytes * 8 / (e0.elapsed_time(e1) * 1e-3) / 1e9
            log(f"read probe: {wgs} workgroups, unroll {unroll}: {gbps:.0f} GB/s")
            if gbps > best[0]:
                best = (gbps, f"{wgs} workgroups, {unroll} loads in flight per thread")
    del buf
    torch.cuda.empty_cache()
    return {"gbps": round(best[0], 1), "buffer": "4 GiB", "launch": best[1],
            "kernel": "delta_hbm_read_probe (16-byte streaming loads)"}


def _graph_us(launch, steps):
    """Per-launch time of `launch()` from a graph of 8 launches replayed `steps` times (after
    two eager launches on a side stream), as the layers are timed."""
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(2):
            launch()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(8):
            launch()
    graph.replay()
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(steps):
        graph.replay()
    e1.record()
    torch.cuda.synchronize()
    return e0.elapsed_time(e1) * 1e3 / (steps * 8)


def gather_ceiling(D, nbytes, steps=20):
    """The time and rate of a plain gather of `nbytes` in random 4 KB chunks (the probe kernel
    of include/delta_probe.h, the page-tile access pattern of the sparse layers) out of a 4 GiB
    buffer, by 256 workgroups, and of a plain streaming read of the same number of contiguous
    bytes (best of a few launch shapes), both timed per launch as the layers are: the floors of
    a sparse layer that moves those bytes, the second one's for any kernel that reads them."""
    span = 4 << 30
    buf = torch.ones(span // 4, dtype=torch.int32, device="cuda")
    n = max(1, int(round(nbytes / 4096)))
    g = torch.Generator().manual_seed(4096)
    chunks = torch.randint(0, span // 4096, (n,), generator=g, dtype=torch.int64).cuda()
    sink = torch.zeros(256 * 256, dtype=torch.int32, device="cuda")
    D.delta_hbm_gather_probe(buf, chunks, sink, 256)   # eager first: checks the chunk indices
    us = _graph_us(lambda: D.delta_hbm_gather_probe(buf, chunks, sink, 256), steps)
    sub = buf[: n * 1024]
    stream = None
    for wgs in (256, 512, 1024):
        for unroll in (4, 8):
            t = _graph_us(lambda: D.delta_hbm_read_probe(sub, sink, wgs, unroll), steps)
            if stream is None or t < stream[0]:
                stream = (t, f"{wgs} workgroups, {unroll} loads in flight per thread")
    del buf, sub
    torch.cuda.empty_cache()
    return {"gbps": round(n * 4096 / (us * 1e-6) / 1e9, 1), "us_per_launch": round(us, 2),
            "bytes": n * 4096, "pattern": "random 4 KB chunks of a 4 GiB buffer, 256 workgroups",
            "kernel": "delta_hbm_gather_probe (16-byte streaming loads, two chunks in flight per thread)",
            "stream_same_bytes": {"us_per_launch": round(stream[0], 2),
                                  "gbps": round(n * 4096 / (stream[0] * 1e-6) / 1e9, 1),
                                  "launch": stream[1],
                                  "kernel": "delta_hbm_read_probe over the same number of contiguous bytes"}}


def time_layers(D, w, sets, stack, shape, sel, ws, steps, other_sel=None):
    """Average duration of one launch of each role's entry point.  For each role, every layer
    of the stack runs that role (its own K/V cache and query), the n launches of one step are
    captured in a HIP graph (one graph per rotating input set), and the graphs are replayed
    `steps` times between two HIP events on the launch stream; per-launch time = elapsed time
    over the number of launches.  Host launch latency and per-call event overhead are excluded;
    the gap between kernels inside a graph is included.  Sparse launches use the selection of
    the Delta layer that precedes them in the schedule (the first Delta layer's for layers
    before it), with its physical pages, as delta_decode_step does.  With `other_sel` (the
    selection parameters with the other Delta-layer path), the Delta role is also timed on that
    path ("delta_other").  Also returns how many layers of the step run each role."""
    roles = stack.roles
    slots, cur = [], -1
    for r in roles:
        if r == configs.ROLE_DELTA:
            cur += 1
        slots.append(cur)

    def step_role(i):
        r = roles[i]
        return "full" if (r == configs.ROLE_FULL or slots[i] < 0) else ROLE_NAME[r]

    counts = {}
    for i in range(len(roles)):
        counts[step_role(i)] = counts.get(step_role(i), 0) + 1
    # every selection slot holds this step's selection and its physical pages
    for i, r in enumerate(roles):
        if r == configs.ROLE_DELTA:
            inp = sets[0]
            kv = D.make_kv(inp.k_cache[i], inp.v_cache[i], inp.page_table, inp.seq_lens)
            D.delta_delta_attn_select(shape, kv, inp.q[i], stack.outs[0][i], sel, stack.sel_idx[slots[i]],
                                      stack.sel_cnt[slots[i]], None, ws, sel_phys=stack.sel_phys[slots[i]])
    torch.cuda.synchronize()
    scratch_idx = torch.empty_like(stack.sel_idx[0])
    scratch_cnt = torch.empty_like(stack.sel_cnt[0])
    scratch_phys = torch.empty_like(stack.sel_phys[0])

    def call(name, si, i):
        inp = sets[si]
        out = stack.outs[si][i]
        kv = D.make_kv(inp.k_cache[i], inp.v_cache[i], inp.page_table, inp.seq_lens)
        if name == "full":
            D.delta_full_attn(shape, kv, inp.q[i], out, ws)
        elif name in ("delta", "delta_other"):
            D.delta_delta_attn_select(shape, kv, inp.q[i], out, sel if name == "delta" else other_sel,
                                      scratch_idx, scratch_cnt, None, ws, sel_phys=scratch_phys)
        else:
            sd = max(slots[i], 0)
            D.delta_sparse_attn(shape, kv, inp.q[i], out, sel, stack.sel_idx[sd], stack.sel_cnt[sd],
                                ws, sel_phys=stack.sel_phys[sd])

    per_role = {}
    for name in ("full", "delta", "sparse") + (("delta_other",) if other_sel is not None else ()):
        if (name if name != "delta_other" else "delta") not in counts:
            continue
        graphs = []
        for si in range(len(sets)):
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                for i in range(len(roles)):
                    call(name, si, i)
            torch.cuda.current_stream().wait_stream(s)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                for i in range(len(roles)):
                    call(name, si, i)
            graphs.append(g)
        for r in range(2):
            graphs[r % len(graphs)].replay()
        torch.cuda.synchronize()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        for r in range(steps):
            graphs[r % len(graphs)].replay()
        e1.record()
        torch.cuda.synchronize()
        per_role[name] = e0.elapsed_time(e1) * 1e3 / (steps * len(roles))
    return per_role, counts


# ------------------------------------------------------------------------------------------
# sweeps over the paper's runtime settings (one JSON line per point, after the headline run's
# protocol: graph-captured steps, inputs resident, rotating input copies below ~1 GiB)
# ------------------------------------------------------------------------------------------
def step_tokens(w, roles, s):
    """Tokens of K/V one DELTA-stack step reads per sequence at context s (for sizing the
    rotation; selection reads at most the budget)."""
    n_dense, seen = 0, False
    for r in roles:
        seen = seen or r == configs.ROLE_DELTA
        n_dense += 1 if (r != configs.ROLE_SPARSE or not seen) else 0
    return n_dense * s + (len(roles) - n_dense) * min(s, w.budget_tokens)


def context_sets(base, s, step_bytes):
    """Input sets at context s (every sequence holding s tokens) over the caches of `base`:
    copy k reads logical pages [k*n, (k+1)*n) of each sequence's pages, so that consecutive
    copies touch disjoint memory; as many copies as bring one round of them past 1 GiB (at
    most 16, and as many as the cached pages hold)."""
    w = base.workload
    n = (s + configs.PAGE - 1) // configs.PAGE
    want = 1 if step_bytes >= (1 << 30) else math.ceil((1 << 30) / max(step_bytes, 1))
    n_rot = max(1, min(16, want, base.max_pages_per_seq // n))
    lens_dev = torch.full((w.batch,), s, dtype=torch.int32, device="cuda")
    sets = []
    for k in range(n_rot):
        pt = torch.zeros_like(base.page_table)
        pt[:, :n] = base.page_table[:, k * n:(k + 1) * n]
        sets.append(synth.DecodeInputs(w, base.k_cache, base.v_cache, base.q, pt, lens_dev,
                                       [s] * w.batch, base.max_pages_per_seq, base.n_phys_pages))
    return sets


def stack_us(D, w, sets, roles, shape, sel, ws, steps, warmup):
    D.delta_workspace_init(ws)
    st = Stack(D, w, sets, roles, shape, sel, ws)
    st.capture()
    us = time_steps(st, steps, warmup) * 1e3
    del st
    return us


def launch_us(D, w, sets, role, shape, sel, ws, steps):
    """Average duration of one launch of the FULL or DELTA entry point on layer 0 of each input
    set, from a graph of one launch per set replayed `steps` times."""
    D.delta_workspace_init(ws)
    K = w.budget_units
    idx = torch.empty((w.batch, K), dtype=torch.int32, device="cuda")
    cnt = torch.empty((w.batch,), dtype=torch.int32, device="cuda")
    phys = torch.empty((w.batch, K), dtype=torch.int32, device="cuda")
    outs = [torch.empty_like(inp.q[0]) for inp in sets]

    def body():
        for inp, out in zip(sets, outs):
            kv = D.make_kv(inp.k_cache[0], inp.v_cache[0], inp.page_table, inp.seq_lens)
            if role == "full":
                D.delta_full_attn(shape, kv, inp.q[0], out, ws)
            else:
                D.delta_delta_attn_select(shape, kv, inp.q[0], out, sel, idx, cnt, None, ws,
                                          sel_phys=phys)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        body()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        body()
    g.replay()
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(steps):
        g.replay()
    e1.record()
    torch.cuda.synchronize()
    return e0.elapsed_time(e1) * 1e3 / (steps * len(sets))


def trapezoid_rounds(points):
    """Sum over decoding rounds 1..S of a per-round time sampled at contexts `points`
    ([(context, us)], ascending, first context 1), by linear interpolation: seconds."""
    tot = 0.0
    for (c0, t0), (c1, t1) in zip(points, points[1:]):
        tot += (t0 + t1) / 2 * (c1 - c0)
    return (tot + points[0][1]) * 1e-6


def emit(rec):
    print(json.dumps(rec), flush=True)


def sweep_rounds(D, w, args):
    """Per-round attention latency while a batch decodes from 1 token to the workload's length
    (the analogue of the paper's per-round latency trace, Sec. 5.3): full stack vs DELTA stack
    at sampled contexts, and the attention time summed over every round."""
    S = w.max_seq_len
    base = synth.make_inputs(w, "cuda", poison_tail=False)
    torch.cuda.synchronize()
    sel = D.make_select(w.budget_tokens, w.recent_tokens, w.unit_tokens, D.DELTA_AGG_MAX)
    ws = D.alloc_workspace(D.make_shape(w.batch, w.n_q_heads, w.n_kv_heads, w.head_dim,
                                        base.max_pages_per_seq, S), sel)
    ctx = sorted({1, 256, 512, w.budget_tokens, w.budget_tokens + configs.PAGE,
                  *range(2048, S + 1, 1024), S})
    full_pts, delta_pts = [], []
    kv_tok = 4 * w.n_kv_heads * w.head_dim
    for s in ctx:
        shape = D.make_shape(w.batch, w.n_q_heads, w.n_kv_heads, w.head_dim,
                             base.max_pages_per_seq, s)
        sets = context_sets(base, s, w.batch * kv_tok * step_tokens(w, w.roles, s))
        full = stack_us(D, w, sets, [configs.ROLE_FULL] * len(w.roles), shape, sel, ws,
                        args.steps, args.warmup)
        delta = stack_us(D, w, sets, w.roles, shape, sel, ws, args.steps, args.warmup)
        full_pts.append((s, full))
        delta_pts.append((s, delta))
        emit({"mode": "rounds", "workload": w.name, "context": s, "full_us": round(full, 2),
              "delta_us": round(delta, 2), "selecting": (s + w.unit_tokens - 1) // w.unit_tokens > w.budget_units,
              "input_copies_rotated": len(sets)})
    tf, td = trapezoid_rounds(full_pts), trapezoid_rounds(delta_pts)
    emit({"mode": "rounds-summary", "workload": w.describe(), "rounds": S,
          "delta_layers": w.delta_layers,
          "attention_s_all_rounds": {"full": round(tf, 3), "delta": round(td, 3)},
          "attention_tokens_per_s": {"full": round(w.batch * S / tf, 1),
                                     "delta": round(w.batch * S / td, 1)},
          "last_round_us": {"full": round(full_pts[-1][1], 2), "delta": round(delta_pts[-1][1], 2)},
          "first_round_us": {"full": round(full_pts[0][1], 2), "delta": round(delta_pts[0][1], 2)}})


class SyntheticDecoder:
    """A decoder with random bf16 weights in the published Qwen2.5-1.5B layout (hidden 1536,
    12 query / 2 KV heads of 128, MLP 8960, vocabulary 151936), wrapped around the attention
    path through delta_decode_step_hooked: before each layer's attention a hook applies the
    RMSNorm and the QKV projection, writes the layer's query and appends the new key and value
    (delta_kv_append, Eq. kv_update); after it, the output projection, the residual, the second
    RMSNorm and the gated MLP.  The round ends with the final norm, the LM head and an argmax.
    Rotary embeddings and projection biases are left out (elementwise work, under 1 % of a
    round).  Everything runs on the step's stream, so a whole round captures into one graph."""

    def __init__(self, D, w, seed=0):
        hid, inter, vocab = 1536, 8960, 151936
        assert (w.n_q_heads * w.head_dim, w.n_kv_heads) == (hid, 2), "Qwen-1.5B attention shape"
        g = torch.Generator(device="cuda").manual_seed(seed)
        dev, bf = "cuda", torch.bfloat16

        def rnd(n_out, n_in):   # [out, in], the layout linear layers keep their weights in
            return (torch.randn((n_out, n_in), generator=g, device=dev) / math.sqrt(n_in)).to(bf)
        L = w.n_layers
        kvd = w.n_kv_heads * w.head_dim
        self.D, self.w = D, w
        self.wqkv = [rnd(hid + 2 * kvd, hid) for _ in range(L)]
        self.wo = [rnd(hid, hid) for _ in range(L)]
        self.wgu = [rnd(2 * inter, hid) for _ in range(L)]
        self.wd = [rnd(hid, inter) for _ in range(L)]
        self.ln1 = [torch.ones(hid, dtype=bf, device=dev) for _ in range(L)]
        self.ln2 = [torch.ones(hid, dtype=bf, device=dev) for _ in range(L)]
        self.lnf = torch.ones(hid, dtype=bf, device=dev)
        self.emb = rnd(vocab, hid)
        self.lm = rnd(vocab, hid)
        self.tokens = torch.randint(0, vocab, (w.batch,), generator=g, device=dev)
        self.x = torch.empty((w.batch, hid), dtype=bf, device=dev)
        self.k_new = torch.empty((w.batch, w.n_kv_heads, w.head_dim), dtype=bf, device=dev)
        self.v_new = torch.empty_like(self.k_new)
        self.next = torch.empty((w.batch,), dtype=torch.int64, device=dev)
        self.hid, self.inter, self.kvd = hid, inter, kvd

    @staticmethod
    def rmsnorm(x, wt, eps=1e-6):
        return torch.nn.functional.rms_norm(x, (x.shape[-1],), wt, eps)

    def hooks(self, inp, outs, shape):
        w, hid, kvd, D = self.w, self.hid, self.kvd, self.D

        def before(i):
            if i == 0:
                self.x.copy_(self.emb.index_select(0, self.tokens))
            lin = torch.nn.functional.linear
            qkv = lin(self.rmsnorm(self.x, self.ln1[i]), self.wqkv[i])
            inp.q[i].view(w.batch, hid).copy_(qkv[:, :hid])
            self.k_new.view(w.batch, kvd).copy_(qkv[:, hid:hid + kvd])
            self.v_new.view(w.batch, kvd).copy_(qkv[:, hid + kvd:])
            D.delta_kv_append(shape, inp.k_cache[i], inp.v_cache[i], inp.page_table,
                              inp.seq_lens, self.k_new, self.v_new)

        def after(i):
            lin = torch.nn.functional.linear
            self.x += lin(outs[i].view(w.batch, hid), self.wo[i])
            gu = lin(self.rmsnorm(self.x, self.ln2[i]), self.wgu[i])
            self.x += lin(torch.nn.functional.silu(gu[:, :self.inter]) * gu[:, self.inter:], self.wd[i])
            if i == w.n_layers - 1:
                logits = lin(self.rmsnorm(self.x, self.lnf), self.lm)
                self.next.copy_(logits.argmax(-1))

        return D.LayerHooks(before=before, after=after)


def sweep_e2e(D, w, args):
    """Whole decoding rounds of a synthetic-weight Qwen-1.5B-shaped model (SyntheticDecoder)
    around the attention path, full attention vs DELTA, over the per-round trace of the
    paper's throughput experiment (Sec. 5.3): per-round latency at sampled contexts, the
    decoding time summed over all rounds, and the throughput."""
    S = w.max_seq_len
    base = synth.make_inputs(w, "cuda", poison_tail=False)
    torch.cuda.synchronize()
    sel = D.make_select(w.budget_tokens, w.recent_tokens, w.unit_tokens, D.DELTA_AGG_MAX)
    ws = D.alloc_workspace(D.make_shape(w.batch, w.n_q_heads, w.n_kv_heads, w.head_dim,
                                        base.max_pages_per_seq, S), sel)
    ctx = sorted({1, 512, w.budget_tokens, w.budget_tokens + configs.PAGE,
                  *range(2048, S + 1, 2048), S})
    kv_tok = 4 * w.n_kv_heads * w.head_dim
    pts = {"full": [], "delta": []}
    model = SyntheticDecoder(D, w)
    for s in ctx:
        shape = D.make_shape(w.batch, w.n_q_heads, w.n_kv_heads, w.head_dim,
                             base.max_pages_per_seq, s)
        sets = context_sets(base, s, w.batch * kv_tok * step_tokens(w, w.roles, s))
        res = {}
        for name, roles in (("full", [configs.ROLE_FULL] * w.n_layers), ("delta", w.roles)):
            D.delta_workspace_init(ws)
            st = Stack(D, w, sets, roles, shape, sel, ws)
            graphs = []
            for k, inp in enumerate(sets):
                hooks = model.hooks(inp, st.outs[k], shape)
                side = torch.cuda.Stream()
                side.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(side):
                    D.delta_decode_step_hooked(st.args[k], hooks)
                torch.cuda.current_stream().wait_stream(side)
                torch.cuda.synchronize()
                gr = torch.cuda.CUDAGraph()
                with torch.cuda.graph(gr):
                    D.delta_decode_step_hooked(st.args[k], hooks)
                graphs.append(gr)
            st.graphs = graphs
            res[name] = time_steps(st, args.steps, args.warmup) * 1e3
            del st, graphs
        for name in pts:
            pts[name].append((s, res[name]))
        emit({"mode": "e2e", "workload": w.name, "context": s, "full_round_us": round(res["full"], 2),
              "delta_round_us": round(res["delta"], 2), "input_copies_rotated": len(sets)})
        torch.cuda.empty_cache()
    tf, td = trapezoid_rounds(pts["full"]), trapezoid_rounds(pts["delta"])
    emit({"mode": "e2e-summary", "workload": w.describe(), "model": "synthetic Qwen2.5-1.5B layout",
          "rounds": S, "delta_layers": w.delta_layers,
          "decode_s_all_rounds": {"full": round(tf, 3), "delta": round(td, 3)},
          "tokens_per_s": {"full": round(w.batch * S / tf, 1), "delta": round(w.batch * S / td, 1)},
          "speedup": round(tf / td, 3),
          "first_round_us": {"full": round(pts["full"][0][1], 1), "delta": round(pts["delta"][0][1], 1)},
          "last_round_us": {"full": round(pts["full"][-1][1], 1), "delta": round(pts["delta"][-1][1], 1)}})


def sweep_deltas(D, w, args):
    """Step time against the number of Delta-layers (Sec. 6.1): at the longest context (the
    last decoding round) and averaged over all rounds 1..S; the full stack alongside."""
    S = w.max_seq_len
    L = w.n_layers
    base = synth.make_inputs(w, "cuda", poison_tail=False)
    torch.cuda.synchronize()
    sel = D.make_select(w.budget_tokens, w.recent_tokens, w.unit_tokens, D.DELTA_AGG_MAX)
    ws = D.alloc_workspace(D.make_shape(w.batch, w.n_q_heads, w.n_kv_heads, w.head_dim,
                                        base.max_pages_per_seq, S), sel)
    ctx = sorted({1, *range(2048, S + 1, 2048), S})
    counts = sorted({1, 2, 3, 4, 6, 8, 12, 16, 20, 24, L - 2} & set(range(1, L - 1)))
    kv_tok = 4 * w.n_kv_heads * w.head_dim
    per_ctx = {}
    for s in ctx:
        shape = D.make_shape(w.batch, w.n_q_heads, w.n_kv_heads, w.head_dim,
                             base.max_pages_per_seq, s)
        # size the rotation for the sparsest schedule, so that no point is served from cache
        sets = context_sets(base, s, w.batch * kv_tok * step_tokens(
            w, configs.roles_for(L, [2]), s))
        full = stack_us(D, w, sets, [configs.ROLE_FULL] * L, shape, sel, ws, args.steps, args.warmup)
        per_ctx[s] = {"full": full}
        for c in counts:
            per_ctx[s][c] = stack_us(D, w, sets, configs.roles_for(L, configs.spread_delta_layers(L, c)),
                                     shape, sel, ws, args.steps, args.warmup)
        log(f"context {s}: full {full:.1f} us, " + ", ".join(f"{c}D {per_ctx[s][c]:.1f}" for c in counts))
    full_avg = trapezoid_rounds([(s, per_ctx[s]["full"]) for s in ctx]) / S * 1e6
    for c in counts:
        avg = trapezoid_rounds([(s, per_ctx[s][c]) for s in ctx]) / S * 1e6
        emit({"mode": "deltas", "workload": w.name, "n_delta": c,
              "delta_layers": configs.spread_delta_layers(L, c),
              "last_round_us": round(per_ctx[S][c], 2), "avg_round_us": round(avg, 2),
              "full_last_round_us": round(per_ctx[S]["full"], 2),
              "full_avg_round_us": round(full_avg, 2)})


def sweep_kl(D, w, args):
    """DELTA step time over a grid of page budgets K and recency windows L (pages; L < K), at
    the workload's context (the runtime counterpart of the paper's (K, L) study, Sec. 6.2)."""
    import dataclasses
    S = w.max_seq_len
    base = synth.make_inputs(w, "cuda", poison_tail=False)
    torch.cuda.synchronize()
    Ks = [32, 64, 128, 256, 512]
    Ls = [1, 2, 4, 8, 16, 32, 64]
    shape = D.make_shape(w.batch, w.n_q_heads, w.n_kv_heads, w.head_dim, base.max_pages_per_seq, S)
    big = D.make_select(configs.PAGE * max(Ks), configs.PAGE, w.unit_tokens, D.DELTA_AGG_MAX)
    ws = D.alloc_workspace(shape, big)
    kv_tok = 4 * w.n_kv_heads * w.head_dim
    sets = context_sets(base, S, w.batch * kv_tok * step_tokens(w, w.roles, S))
    sel0 = D.make_select(w.budget_tokens, w.recent_tokens, w.unit_tokens, D.DELTA_AGG_MAX)
    full = stack_us(D, w, sets, [configs.ROLE_FULL] * w.n_layers, shape, sel0, ws, args.steps, args.warmup)
    for K in Ks:
        for Lp in (l for l in Ls if l < K):
            wk = dataclasses.replace(w, budget_tokens=configs.PAGE * K, recent_pages=Lp)
            sel = D.make_select(wk.budget_tokens, wk.recent_tokens, wk.unit_tokens, D.DELTA_AGG_MAX)
            us = stack_us(D, wk, sets, wk.roles, shape, sel, ws, args.steps, args.warmup)
            emit({"mode": "kl", "workload": w.name, "context": S, "K_pages": K, "L_pages": Lp,
                  "delta_us": round(us, 2), "full_us": round(full, 2),
                  "speedup": round(full / us, 3)})


def sweep_overhead(D, args):
    """Delta-layer overhead over a full layer against context length, per model shape on one
    GPU without tensor parallelism (the analogue of the paper's kernel breakdown, App. E):
    per-launch time of the DELTA entry point (attention + logits, scoring, selection) and of
    the FULL entry point, over a 1k-token budget."""
    shapes = [("qwen1.5b", 12, 2, 64), ("qwen7b", 28, 4, 64), ("qwen14b", 40, 8, 32)]
    ctx = [1024, 2048, 4096, 8192, 16384, 32768]
    for name, hq, hkv, B in shapes:
        w = configs.Workload(9, f"{name}-b{B}-layer", 1, hq, hkv, 128, B, max(ctx), 1024,
                             hh_frac=0.02, hh_factor=4.0, recent_pages=8,
                             roles=[configs.ROLE_DELTA])
        base = synth.make_inputs(w, "cuda", poison_tail=False)
        torch.cuda.synchronize()
        sel = D.make_select(w.budget_tokens, w.recent_tokens, w.unit_tokens, D.DELTA_AGG_MAX)
        ws = D.alloc_workspace(D.make_shape(B, hq, hkv, 128, base.max_pages_per_seq, max(ctx)), sel)
        for s in ctx:
            shape = D.make_shape(B, hq, hkv, 128, base.max_pages_per_seq, s)
            sets = context_sets(base, s, B * s * 4 * hkv * 128)
            f = launch_us(D, w, sets, "full", shape, sel, ws, args.steps)
            d = launch_us(D, w, sets, "delta", shape, sel, ws, args.steps)
            emit({"mode": "overhead", "shape": f"{name} Hq/Hkv/d={hq}/{hkv}/128 B={B}",
                  "context": s, "full_us": round(f, 2), "delta_us": round(d, 2),
                  "overhead": round((d - f) / f, 4), "input_copies_rotated": len(sets)})
        del base, ws
        torch.cuda.empty_cache()


def sweep_append(D, w, args):
    """Decode-step integration (Eq. kv_update): the KV append's per-launch time, and the DELTA
    step with every layer's append enqueued by a before-attention hook of
    delta_decode_step_hooked, against the same step without appends (both graph-captured)."""
    lens = synth.seq_lens_for(w)
    # the appended token is the last one counted by seq_lens, so the step reads it
    sets = build_sets(w, 1)
    inp = sets[0]
    shape = D.make_shape(w.batch, w.n_q_heads, w.n_kv_heads, w.head_dim, inp.max_pages_per_seq,
                         inp.max_seq_len)
    sel = D.make_select(w.budget_tokens, w.recent_tokens, w.unit_tokens, D.DELTA_AGG_MAX)
    ws = D.alloc_workspace(shape, sel)
    g = torch.Generator(device="cuda").manual_seed(1)
    k_new = [torch.randn((w.batch, w.n_kv_heads, w.head_dim), generator=g, device="cuda").to(torch.bfloat16)
             for _ in range(w.n_layers)]
    v_new = [torch.randn_like(k, dtype=torch.float32).to(torch.bfloat16) for k in k_new]

    def append(i):
        D.delta_kv_append(shape, inp.k_cache[i], inp.v_cache[i], inp.page_table, inp.seq_lens,
                          k_new[i], v_new[i])

    def graph_of(fn):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            fn()
        torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            fn()
        return gr

    def timed(gr, steps):
        for _ in range(3):
            gr.replay()
        torch.cuda.synchronize()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        for _ in range(steps):
            gr.replay()
        e1.record()
        torch.cuda.synchronize()
        return e0.elapsed_time(e1) * 1e3 / steps

    us_append = timed(graph_of(lambda: [append(i) for i in range(w.n_layers)]), args.steps) / w.n_layers
    st = Stack(D, w, sets, w.roles, shape, sel, ws)
    hooks = D.LayerHooks(before=append)
    plain = graph_of(lambda: D.delta_decode_step(st.args[0]))
    hooked = graph_of(lambda: D.delta_decode_step_hooked(st.args[0], hooks))
    us_plain = timed(plain, args.steps)
    us_hooked = timed(hooked, args.steps)
    moved = 4 * w.batch * w.n_kv_heads * w.head_dim * 2   # read k/v_new, write the two rows
    emit({"mode": "append", "workload": w.describe(), "append_us_per_launch": round(us_append, 2),
          "append_bytes_per_launch": moved, "delta_step_us": round(us_plain, 2),
          "delta_step_with_append_hooks_us": round(us_hooked, 2),
          "append_share_of_step": round((us_hooked - us_plain) / us_plain, 4),
          "seq_lens_max": max(lens)})


# ------------------------------------------------------------------------------------------
def cpu_baseline(w, inp, roles, budget_s):
    """The oracle as it stands, on this host: gather + every layer of the DELTA-stack step for
    whole sequences, until `budget_s` seconds are spent; scaled to microseconds per step."""
    import numpy as np
    from oracle import delta_oracle as O
    try:
        import threadpoolctl
        threads = max([p.get("num_threads", 1) for p in threadpoolctl.threadpool_info()] or [1])
    except Exception:   # pragma: no cover
        threads = 1
    scale = O.default_scale(w.head_dim)
    done, spent, toks = 0, 0.0, 0
    for b in range(w.batch):
        host = [synth.sequence_pages(inp, i, b) for i in range(len(roles))]
        qs = [O.bf16_bits_to_f64(synth.bits(inp.q[i][b])) for i in range(len(roles))]
        s_b = inp.seq_lens_host[b]
        t = time.perf_counter()
        ident = np.arange(host[0][0].shape[0])
        Ks = [O.gather_tokens(kb, ident, s_b) for kb, _ in host]
        Vs = [O.gather_tokens(vb, ident, s_b) for _, vb in host]
        O.decode_step_sequence(roles, qs, Ks, Vs, scale, w.unit_tokens, w.budget_units,
                               w.recent_units)
        spent += time.perf_counter() - t
        done += 1
        toks += s_b
        del host, Ks, Vs
        if spent >= budget_s:
            break
    # the oracle's work grows linearly with a sequence's length: scale by tokens
    total = sum(inp.seq_lens_host)
    us_per_step = spent / toks * total * 1e6
    sample = (f"oracle DELTA-stack step (gather + {len(roles)} layers) of {done} of {w.batch} "
              f"sequence(s) ({toks} of {total} tokens), {spent:.1f} s; the per-step value is "
              f"extrapolated linearly per token" if done < w.batch else
              f"oracle DELTA-stack step (gather + {len(roles)} layers) of all {w.batch} "
              f"sequence(s), {spent:.1f} s")
    # oracle seconds per (sequence, layer) for each role, on sequence 0's first layer
    host = synth.sequence_pages(inp, 0, 0)
    s0 = inp.seq_lens_host[0]
    ident = np.arange(host[0].shape[0])
    K0, V0 = O.gather_tokens(host[0], ident, s0), O.gather_tokens(host[1], ident, s0)
    q0 = O.bf16_bits_to_f64(synth.bits(inp.q[0][0]))
    per_role = {}
    t = time.perf_counter()
    _, alpha = O.full_attention(q0, K0, V0, scale)
    per_role["full"] = time.perf_counter() - t
    t = time.perf_counter()
    _, alpha = O.full_attention(q0, K0, V0, scale)
    rho, _ = O.refresh_units(alpha, w.unit_tokens, w.budget_units, w.recent_units)
    per_role["delta"] = time.perf_counter() - t
    t = time.perf_counter()
    O.sparse_attention(q0, K0, V0, rho, w.unit_tokens, scale)
    per_role["sparse"] = time.perf_counter() - t
    model = ""
    try:
        for line in open("/proc/cpuinfo"):
            if line.startswith("model name"):
                model = line.split(":", 1)[1].strip()
                break
    except OSError:   # pragma: no cover
        pass
    return {"value": us_per_step, "unit": "us/step", "cores": threads, "kind": "oracle",
            "sample": sample, "host_cpus": len(os.sched_getaffinity(0)), "cpu_model": model,
            "seconds_per_sequence_layer": {k: round(v, 4) for k, v in per_role.items()}}


ATTN_SOURCES = ("attn_kernel.hip", "attn_tile.h", "wave.h")


def attn_source_sha256():
    """sha256 over the attention kernel's source files, in ATTN_SOURCES order."""
    import hashlib
    h = hashlib.sha256()
    for f in ATTN_SOURCES:
        h.update(open(os.path.join(ROOT, "paper_2510_09883_amd", "csrc", f), "rb").read())
    return h.hexdigest()


def measured_traffic(role, w, kernel_tag):
    """HBM bytes per launch of the dominant kernel from the committed rocprofv3 counter summary
    (FETCH_SIZE + WRITE_SIZE, scaled by a known-size copy), or None when there is none for this
    kernel and workload or the kernel source has changed since the counters were taken."""
    path = os.path.join(ROOT, "profiles", f"attn_{role}_{w.name}.md")
    if not os.path.exists(path):
        return None
    kv = {}
    for line in open(path):
        if ":" in line:
            k, v = line.split(":", 1)
            kv[k.strip()] = v.strip()
    if kv.get("kernel") != kernel_tag:
        return None
    if kv.get("source_sha256") != attn_source_sha256():
        return None
    return int(kv["traffic_bytes_per_launch"])


def copy_calibration():
    """A plain device copy of known size (64 MiB read + 64 MiB written), for scaling the
    FETCH_SIZE / WRITE_SIZE counters of the profiled kernels."""
    a = torch.empty(64 << 20, dtype=torch.uint8, device="cuda").fill_(1)
    b = torch.empty_like(a)
    torch.cuda.synchronize()
    b.copy_(a)
    torch.cuda.synchronize()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--gpus", type=int, default=1)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--warmup", type=int, default=5)
    # default: the largest single-GPU workload, the Llama-8B shape over a ragged batch of 32
    # sequences of 16K-32K tokens on a shuffled page table (~103 GB of KV resident), the
    # stand-in for the paper's large-batch long-decoding runtime setting
    ap.add_argument("--config", type=int, default=None, choices=list(range(1, 9)),
                    help="workload (default 5; the sweeps default to the paper's model for them)")
    ap.add_argument("--delta-layers", type=str, default=None,
                    help="comma-separated Delta-layer indices replacing the workload's schedule")
    ap.add_argument("--sweep", choices=["rounds", "deltas", "kl", "overhead", "append", "e2e"], default=None,
                    help="print one JSON line per point of a runtime sweep instead of the "
                         "headline measurement")
    ap.add_argument("--unit-tokens", type=int, default=16, choices=[16, 1])
    ap.add_argument("--cpu-seconds", type=float, default=20.0)
    ap.add_argument("--no-cpu-baseline", action="store_true")
    args = ap.parse_args()
    if args.gpus != 1 or int(os.environ.get("WORLD_SIZE", "1")) != 1:
        print("bench.py runs on exactly one GPU: this library has no multi-GPU path "
              "(--gpus must be 1).", file=sys.stderr)
        sys.exit(2)
    from paper_2510_09883_amd import delta as D

    if args.sweep is not None:
        default = {"rounds": 6, "deltas": 6, "kl": 7, "overhead": None, "append": 3, "e2e": 6}[args.sweep]
        w = configs.get(args.config or default, args.unit_tokens) if default else None
        if w is not None and args.delta_layers:
            w.set_delta_layers(args.delta_layers.split(","))
        if w is not None:
            log(f"sweep {args.sweep}: {w.describe()}")
        {"rounds": lambda: sweep_rounds(D, w, args), "deltas": lambda: sweep_deltas(D, w, args),
         "kl": lambda: sweep_kl(D, w, args), "overhead": lambda: sweep_overhead(D, args),
         "append": lambda: sweep_append(D, w, args), "e2e": lambda: sweep_e2e(D, w, args)}[args.sweep]()
        return

    w = configs.get(args.config or 5, args.unit_tokens)
    if args.delta_layers:
        w.set_delta_layers(args.delta_layers.split(","))
    lens = synth.seq_lens_for(w)
    fb = full_layer_bytes(w, lens)
    n_delta = sum(r == configs.ROLE_DELTA for r in w.roles)
    n_sets = 1
    approx_delta_step = (len(w.roles) - n_delta) * fb * min(1.0, w.budget_tokens / max(lens)) + n_delta * fb
    if approx_delta_step < (1 << 30):
        n_sets = min(8, 1 + math.ceil((1 << 30) / approx_delta_step))
    sets = build_sets(w, n_sets)
    inp = sets[0]
    shape = D.make_shape(w.batch, w.n_q_heads, w.n_kv_heads, w.head_dim, inp.max_pages_per_seq,
                         inp.max_seq_len)
    sel = D.make_select(w.budget_tokens, w.recent_tokens, w.unit_tokens, D.DELTA_AGG_MAX)
    ws = D.alloc_workspace(shape, sel)

    delta_stack = Stack(D, w, sets, w.roles, shape, sel, ws)
    full_stack = Stack(D, w, sets, [configs.ROLE_FULL] * len(w.roles), shape, sel, ws)
    delta_stack.capture()
    full_stack.capture()
    log("graphs captured")

    ms_full = time_steps(full_stack, args.steps, args.warmup)
    ms_delta = time_steps(delta_stack, args.steps, args.warmup)
    log(f"full stack {ms_full * 1e3:.1f} us/step, DELTA stack {ms_delta * 1e3:.1f} us/step")
    dist = {"delta": step_distribution(delta_stack, args.steps),
            "full": step_distribution(full_stack, args.steps)}

    # algorithmic bytes of one DELTA step from the selections it made
    idx = delta_stack.sel_idx.cpu().numpy()
    cnt = delta_stack.sel_cnt.cpu().numpy()
    slot = -1
    delta_bytes = 0
    sparse_bytes = []
    for r in w.roles:
        if r == configs.ROLE_DELTA:
            slot += 1
        if r == configs.ROLE_SPARSE and slot >= 0:
            sb = sparse_layer_bytes(w, lens, idx[slot], cnt[slot])
            sparse_bytes.append(sb)
            delta_bytes += sb
        else:
            delta_bytes += fb
    full_bytes = fb * len(w.roles)

    # the Delta-layer path the step takes (DELTA_PATH_AUTO), and the other path timed beside it
    # where both can run on this workload
    step_fused = D.delta_delta_path(shape, sel)
    other_sel = D.make_select(w.budget_tokens, w.recent_tokens, w.unit_tokens, D.DELTA_AGG_MAX,
                              D.DELTA_PATH_SPLIT if step_fused else D.DELTA_PATH_FUSED)
    if configs.ROLE_DELTA not in w.roles or D.delta_delta_path(shape, other_sel) == step_fused:
        other_sel = None
    layer_us, per_step = time_layers(D, w, sets, delta_stack, shape, sel, ws, args.steps, other_sel)
    other_us = layer_us.pop("delta_other", None)
    log(f"per-launch us: {layer_us}, Delta path {'fused' if step_fused else 'split'}" +
        (f", other path {other_us:.2f}" if other_us else ""))
    sb_avg = sum(sparse_bytes) / len(sparse_bytes) if sparse_bytes else 0
    role_bytes = {"full": fb, "delta": fb, "sparse": sb_avg}
    dominant = max(layer_us, key=lambda r: layer_us[r] * per_step[r])
    kernel_name = {"full": "attn_kernel (dense rows)", "delta": "attn_kernel + score + select",
                   "sparse": "attn_kernel (selected pages)"}[dominant]
    mode = {"full": 0, "delta": 0, "sparse": 1 if w.unit_tokens == 16 else 2}[dominant]
    logits = "true" if dominant == "delta" else "false"
    # dense launches over 2-64 sequences run the balanced instantiation
    balanced = "true" if mode == 0 and 2 <= w.batch <= 64 else "false"
    kernel_tag = f"attn_kernel<{w.head_dim}, {w.group}, {mode}, {logits}, {balanced}, false>"   # bf16 caches
    traffic = measured_traffic(dominant, w, kernel_tag)
    achieved = role_bytes[dominant] / (layer_us[dominant] * 1e-6) / 1e9
    overhead = (layer_us["delta"] - layer_us["full"]) / layer_us["full"] if "delta" in layer_us and "full" in layer_us else None

    ceiling = read_ceiling(D)
    log(f"measured read ceiling {ceiling}")
    gather = gather_ceiling(D, sb_avg) if sb_avg else None
    log(f"gather of the sparse layer's bytes: {gather}")

    cpu = None
    if not args.no_cpu_baseline:
        log("timing the CPU oracle")
        cpu = cpu_baseline(w, inp, w.roles, args.cpu_seconds)

    copy_calibration()

    us_delta = ms_delta * 1e3
    rec = {
        "metric": METRIC,
        "value": round(us_delta, 2),
        "unit": "us/step",
        "n_gpus": 1,
        "steps": args.steps,
        "warmup": args.warmup,
        "ms_per_step": round(ms_delta, 5),
        "higher_is_better": False,
        "scaling": "weak",
        "vs_baseline": None,
        "dtype": "bf16",
        "accum": "fp32",
        "data": "synthetic",
        "config": {
            "workload": w.describe(),
            "batch": w.batch, "seq_len": w.max_seq_len, "layers": len(w.roles),
            "budget_tokens": w.budget_tokens, "recent_tokens": w.recent_tokens,
            "unit_tokens": w.unit_tokens,
            "delta_layers": [i for i, r in enumerate(w.roles) if r == configs.ROLE_DELTA],
            "input_copies_rotated": n_sets, "graph": True,
        },
        "full_stack_us_per_step": round(ms_full * 1e3, 2),
        "step_us_distribution": dist,
        "delta_speedup_vs_full": round(ms_full / ms_delta, 3),
        "tokens_per_s": {"delta": round(w.batch / (ms_delta * 1e-3), 1),
                         "full": round(w.batch / (ms_full * 1e-3), 1)},
        "hbm_gbps_algorithmic": {"delta_stack": round(delta_bytes / (ms_delta * 1e-3) / 1e9, 1),
                                 "full_stack": round(full_bytes / (ms_full * 1e-3) / 1e9, 1)},
        "frac_of_peak": {"delta_stack": round(delta_bytes / (ms_delta * 1e-3) / 1e9 / HBM_PEAK_GBPS, 4),
                         "full_stack": round(full_bytes / (ms_full * 1e-3) / 1e9 / HBM_PEAK_GBPS, 4)},
        "layer_us": {k: round(v, 2) for k, v in layer_us.items()},
        "layer_gbps": {k: round(role_bytes[k] / (layer_us[k] * 1e-6) / 1e9, 1) for k in layer_us},
        "layer_frac_of_peak": {k: round(role_bytes[k] / (layer_us[k] * 1e-6) / 1e9 / HBM_PEAK_GBPS, 4)
                               for k in layer_us},
        "measured_read_ceiling": ceiling,
        "layer_frac_of_measured_ceiling": {k: round(role_bytes[k] / (layer_us[k] * 1e-6) / 1e9 / ceiling["gbps"], 4)
                                           for k in layer_us},
        "sparse_gather_floor": None if gather is None or "sparse" not in layer_us else dict(
            gather, sparse_layer_over_floor=round(layer_us["sparse"] / gather["us_per_launch"], 4),
            sparse_layer_over_stream=round(layer_us["sparse"] / gather["stream_same_bytes"]["us_per_launch"], 4)),
        "delta_select_overhead": None if overhead is None else round(overhead, 4),
        "delta_path": None if configs.ROLE_DELTA not in w.roles else ("fused" if step_fused else "split"),
        "delta_other_path": None if other_us is None else {
            "path": "split" if step_fused else "fused",
            "note": ("the Delta layer on the path the step does not take (DELTA_PATH_AUTO takes the "
                     "fused kernel where its grid of one workgroup per 64-page chunk and sequence "
                     "fills the device and is resident at once), timed the same way"),
            "grid_workgroups_fused": w.batch * math.ceil(math.ceil(max(lens) / 16) / 64),
            "layer_us": round(other_us, 2),
            "delta_select_overhead": round((other_us - layer_us["full"]) / layer_us["full"], 4)},
        "roofline": {"bound": "hbm", "kernel": kernel_name, "achieved": round(achieved, 1),
                     "peak": HBM_PEAK_GBPS, "unit": "GB/s", "frac": round(achieved / HBM_PEAK_GBPS, 4),
                     "traffic": traffic, "bytes_per_launch": int(role_bytes[dominant]),
                     "avg_launch_us": round(layer_us[dominant], 3)},
        "cpu_baseline": cpu,
        "paper_context": PAPER_CONTEXT,
    }
    print(json.dumps(rec), flush=True)


if __name__ == "__main__":
    main()
