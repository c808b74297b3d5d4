"""The operators around the cache as a server runs them: prompts are rotated, appended and attended in
chunks, drafted tokens are verified at once, and a decoding step with the three layer roles goes on
from there, for bf16 and e4m3 caches; the debug build's checks of the same calls."""
import ctypes
import os

import pytest
import torch

from cache_cases import PAGE, attend, default_scale, worst
from gpu_helpers import D
from test_gpu_rope_append import frequencies, rotated

pytestmark = pytest.mark.gpu

HQ, HKV, HD = 14, 2, 128
P_ROUND = 2.0 ** -8


def E():
    from paper_2510_09883_amd import extend
    return extend


class Server:
    """One layer's cache of three sequences that grow, and the calls that a server makes."""

    def __init__(self, e4m3, capacity=704):
        self.B, self.width = 3, capacity // PAGE
        g = torch.Generator().manual_seed(1)
        self.g = torch.Generator().manual_seed(2)
        kind = torch.float8_e4m3fn if e4m3 else torch.bfloat16
        n = self.B * self.width
        self.table = torch.randperm(n, generator=g).int().view(self.B, self.width)
        self.caches = [torch.full((n, HKV, PAGE, HD), float("nan")).to(kind).cuda() for _ in range(2)]
        self.scales = [(0.02 + 0.05 * torch.rand((HKV,), generator=g)).cuda() for _ in range(2)] if e4m3 else [None, None]
        self.lens = torch.zeros((self.B,), dtype=torch.int32, device="cuda")
        self.table_gpu = self.table.cuda()
        self.kv = D().make_kv(*self.caches, self.table_gpu, self.lens, *self.scales)
        self.shape = D().make_shape(self.B, HQ, HKV, HD, self.width, capacity)
        self.inv_freq = frequencies(HD, 1e6)
        self.inv_freq_gpu = self.inv_freq.cuda()

    def feed(self, new):
        """New tokens of every sequence through append and attention: (inputs, rotated queries, outputs)."""
        rows = sum(new)
        qkv = torch.randn((rows, HQ + 2 * HKV, HD), generator=self.g).to(torch.bfloat16)
        dev = qkv.cuda()
        offsets = torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32).cuda()
        self.lens += torch.tensor(new, dtype=torch.int32).cuda()
        q = torch.full((rows, HQ, HD), float("nan"), dtype=torch.bfloat16, device="cuda")
        out = torch.full_like(q, float("nan"))
        E().delta_rope_append(self.shape, self.kv, dev[:, :HQ], dev[:, HQ:HQ + HKV], dev[:, HQ + HKV:], q,
                              self.inv_freq_gpu, row_offsets=offsets)
        ws = E().alloc_extend_workspace(self.shape, rows, max(new))
        E().delta_extend_attn(self.shape, self.kv, q, out, offsets, max(new), ws)
        torch.cuda.synchronize()
        return qkv, q.cpu(), out.cpu()

    def tokens(self, which, b, n):
        """float64 [n, hkv, d] of what the cache holds for sequence b's first n tokens."""
        t = torch.arange(n)
        x = self.caches[which].cpu().double()[self.table[b, t // PAGE].long(), :, t % PAGE]
        return x if self.scales[which] is None else x * self.scales[which].cpu().double()[:, None]

    def check(self, new, q, out, pick=lambda n: range(n)):
        row = 0
        for b, n in enumerate(new):
            s = int(self.lens[b])
            k, v = self.tokens(0, b, s), self.tokens(1, b, s)
            for j in pick(n):
                m = s - n + j + 1
                want, tol = attend(q[row + j], k[:m], v[:m], default_scale(HD), P_ROUND)
                assert worst(out[row + j], want, tol) <= 1, f"row {j} of sequence {b}"
            row += n


@pytest.mark.parametrize("e4m3", [False, True])
def test_prompts_chunks_drafts_and_a_decoding_step(e4m3):
    d = D()
    srv = Server(e4m3)
    new = [300, 17, 1]
    qkv, q, out = srv.feed(new)          # prompts
    srv.check(new, q, out, lambda n: sorted({0, n - 1, n // 2, n // 3}))
    # the cache holds the rotated keys and the values of these very inputs
    row = 0
    for b, n in enumerate(new):
        k, tol = rotated(qkv[row:row + n, HQ:HQ + HKV], torch.arange(n), srv.inv_freq, False)
        held = srv.tokens(0, b, n)
        unit = srv.scales[0].cpu().double()[:, None] if e4m3 else torch.ones((HKV, 1), dtype=torch.float64)
        half = torch.maximum(k.abs() * 2.0 ** -4, unit * 2.0 ** -10) if e4m3 else k.abs() * 2.0 ** -8
        assert bool(((held - k).abs() <= half * (1 + 2.0 ** -10) + tol).all())
        row += n
    for new in ([200, 0, 64], [0, 300, 128]):   # the next chunks
        _, q, out = srv.feed(new)
        srv.check(new, q, out, lambda n: sorted({0, n - 1, n // 2} if n else ()))
    new = [5, 1, 8]                       # drafted tokens
    _, q, out = srv.feed(new)
    srv.check(new, q, out)

    # one decoding step: every layer has this cache; its token is appended first
    srv.lens += 1
    qkv = torch.randn((3, HQ + 2 * HKV, HD), generator=srv.g).to(torch.bfloat16).cuda()
    roles = [d.DELTA_ROLE_FULL, d.DELTA_ROLE_DELTA, d.DELTA_ROLE_SPARSE]
    qs = [torch.empty((3, HQ, HD), dtype=torch.bfloat16, device="cuda") for _ in roles]
    outs = [torch.full_like(x, float("nan")) for x in qs]
    sel = d.make_select(128, 16)
    idx = torch.zeros((1, 3, 8), dtype=torch.int32, device="cuda")
    cnt = torch.zeros((1, 3), dtype=torch.int32, device="cuda")
    args = d.StepArgs(srv.shape, roles, [srv.kv] * 3, qs, outs, sel, idx, cnt, d.alloc_workspace(srv.shape, sel))

    def before(i):
        E().delta_rope_append(srv.shape, srv.kv, qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], qs[i],
                              srv.inv_freq_gpu)
    d.delta_decode_step_hooked(args, d.LayerHooks(before=before))
    torch.cuda.synchronize()
    single = torch.full_like(outs[0], float("nan"))
    E().delta_extend_attn(srv.shape, srv.kv, qs[0], single, None, 1, E().alloc_extend_workspace(srv.shape, 3, 1))
    torch.cuda.synchronize()
    for b in range(3):
        s = int(srv.lens[b])
        k, v = srv.tokens(0, b, s), srv.tokens(1, b, s)
        want, tol = attend(qs[0][b].cpu(), k, v, default_scale(HD))
        assert worst(outs[0][b], want, tol) <= 1 and worst(outs[1][b], want, tol) <= 1
        want1, tol1 = attend(qs[0][b].cpu(), k, v, default_scale(HD), P_ROUND)
        assert worst(single[b], want1, tol1) <= 1
        t = (idx[0, b, :int(cnt[0, b])].cpu()[:, None] * PAGE + torch.arange(PAGE)).flatten()
        t = t[t < s]
        want, tol = attend(qs[2][b].cpu(), k[t], v[t], default_scale(HD))
        assert worst(outs[2][b], want, tol) <= 1


def test_two_streams_and_captured_steps():
    """Two servers on streams of their own, each with its workspace, captured once and replayed in turn
    with their eager selves between the replays."""
    servers, graphs, want = [], [], []
    for i, e4m3 in enumerate((False, True)):
        srv = Server(e4m3)
        srv.feed([300, 200, 100])
        new = [3, 1, 2]
        srv.lens += torch.tensor(new, dtype=torch.int32).cuda()
        dev = torch.randn((6, HQ + 2 * HKV, HD), generator=srv.g).to(torch.bfloat16).cuda()
        off = torch.tensor([0, 3, 4, 6], dtype=torch.int32).cuda()
        q, out = (torch.zeros((6, HQ, HD), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ws = E().alloc_extend_workspace(srv.shape, 6, 3)

        def step(srv=srv, dev=dev, off=off, q=q, out=out, ws=ws):
            E().delta_rope_append(srv.shape, srv.kv, dev[:, :HQ], dev[:, HQ:HQ + HKV], dev[:, HQ + HKV:], q,
                                  srv.inv_freq_gpu, row_offsets=off)
            E().delta_extend_attn(srv.shape, srv.kv, q, out, off, 3, ws)
        step()
        torch.cuda.synchronize()
        want.append(out.clone())
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            step()
        servers.append((step, out, stream))
        graphs.append(graph)
    for _ in range(3):
        for step, out, _ in servers:
            out.zero_()
        torch.cuda.synchronize()
        for graph, (_, _, stream) in zip(graphs, servers):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for (step, out, _), w in zip(servers, want):
            assert torch.equal(out, w)
            out.zero_()
            step()
        torch.cuda.synchronize()
        for (_, out, _), w in zip(servers, want):
            assert torch.equal(out, w)


DBG = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                   "paper_2510_09883_amd", "libdelta_attn_debug.so")


@pytest.fixture
def dbg(monkeypatch):
    if not os.path.exists(DBG):
        pytest.skip("the debug library is not built (python -m paper_2510_09883_amd.build --debug)")
    lib = E()._bind(D()._bind(ctypes.CDLL(DBG)))
    monkeypatch.setattr(D(), "_lib", lib)
    return D()


@pytest.mark.parametrize("e4m3", [False, True])
def test_debug_build_gives_the_same_results(dbg, e4m3):
    srv = Server(e4m3)
    for new in ([70, 1, 40], [2, 3, 0]):
        _, q, out = srv.feed(new)
        srv.check(new, q, out)


def test_debug_build_flags_pages_past_the_cache(dbg):
    """The descriptor states fewer pages than the buffers have, so that the bad entry stays inside them:
    attention flags it and reads page 0, the append leaves the token out."""
    srv = Server(False)
    srv.feed([40, 20, 10])
    n = int(srv.table.max())
    bad = next((b, p) for b in range(3) for p in range(srv.width) if int(srv.table[b, p]) == n)
    before = [c.clone() for c in srv.caches]
    srv.kv.n_pages = n          # the last page is past the cache now
    b, page = bad
    srv.lens[b] = 16 * page + 1
    q = torch.zeros((3, HQ, HD), dtype=torch.bfloat16, device="cuda")
    k = torch.ones((3, HKV, HD), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)
    E().delta_rope_append(srv.shape, srv.kv, None, k, k, None)
    ws = E().alloc_extend_workspace(srv.shape, 3, 1)
    E().delta_extend_attn(srv.shape, srv.kv, q, out, None, 1, ws)
    torch.cuda.synchronize()
    assert int(ws[:4].view(torch.int32)[0]) & dbg.DELTA_DEBUG_PAGE
    for c, w in zip(srv.caches, before):
        assert torch.equal(c[n].view(torch.int16), w[n].view(torch.int16))
