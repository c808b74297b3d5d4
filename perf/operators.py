"""Timed cases of the operators around the paged KV cache: filling it with rotated keys, decode
attention over a cache of 8-bit values, and attention of runs of new tokens.

`kind` "append": `delta_rope_append` rotates the queries and keys of ragged runs of new tokens and
writes keys and values into the paged cache.  "full" and "sparse": `delta_full_attn` and
`delta_sparse_attn` over an e4m3 cache.  "extend": `delta_extend_attn`, causal attention of every
new token of ragged runs over the cached tokens up to itself.

Plain values of a case: heads `hq`/`hkv`, head size `d`, `batch` sequences that hold `lo`..`hi`
tokens (drawn uniformly, one of them `hi`), of which `new_lo`..`new_hi` are new (`singles`: only the
first sequence has a run, the others one new token each), `kv8` (e4m3 cache with one scale per KV
head, else bf16), `pad` rows behind the last run, `packed` (q, k and v are views of one projection's
output), `rot` rotated values per head, `interleaved` pairs, `budget` tokens of a sparse layer.
"""
import math

import torch

own = False

PAGE = 16

# Head layouts of the models in paper_2510_09883_amd/configs.py (and rank shares of them)
LLAMA_8B = dict(hq=32, hkv=8, d=128)
QWEN_7B = dict(hq=28, hkv=4, d=128)
QWEN_14B = dict(hq=40, hkv=8, d=128)
QWEN_1_5B = dict(hq=12, hkv=2, d=128)
QWEN_14B_QUARTER = dict(hq=10, hkv=2, d=128)
SMALL = dict(hq=8, hkv=2, d=64)
MODELS = [LLAMA_8B, QWEN_7B, QWEN_14B, QWEN_1_5B, QWEN_14B_QUARTER, SMALL]


def _case(kind, model, batch, lo, hi, new_lo=1, new_hi=1, **kw):
    c = dict(kind=kind, **model, batch=batch, lo=lo, hi=hi, new_lo=new_lo, new_hi=new_hi,
             singles=False, kv8=False, pad=0, packed=True, rot=model["d"], interleaved=False, budget=2048)
    c.update(kw)
    return c


def listed():
    return [
        # one user's decoding round: one token, where only latency counts
        _case("append", QWEN_7B, 1, 4096, 4096, name="append-1x1"),
        # a decoding round of a large batch into an 8-bit cache
        _case("append", QWEN_1_5B, 64, 600, 1500, name="append-64x1-8bit", kv8=True),
        # a batch of prompts as a server collects them, padded behind the last one
        _case("append", LLAMA_8B, 4, 700, 2900, 700, 2900, name="append-4-prompts", pad=37),
        # long prompts into an 8-bit cache, a partly rotated head of interleaved pairs
        _case("append", QWEN_14B, 3, 20000, 32768, 20000, 32768, name="append-3x32k-8bit", kv8=True,
              packed=False, rot=64, interleaved=True),
        # a full layer over an 8-bit cache for one user far into a long decode
        _case("full", QWEN_7B, 1, 32768, 32768, name="full8-1x32k", kv8=True),
        # the same of the library's main workload: 32 ragged sequences of 16K-32K tokens
        _case("full", LLAMA_8B, 32, 16384, 32768, name="full8-32x32k", kv8=True),
        # the sparse layer over an 8-bit cache
        _case("sparse", LLAMA_8B, 16, 32768, 32768, name="sparse8-16x32k", kv8=True, budget=4096),
        # short ragged prompts of a small model, some of one token, some of none
        _case("extend", SMALL, 8, 0, 300, 0, 300, name="extend-8-short"),
        # drafted tokens of a batch, verified at once
        _case("extend", LLAMA_8B, 16, 4000, 16384, 1, 8, name="extend-16x8-drafts"),
        # one long prompt
        _case("extend", LLAMA_8B, 1, 8192, 8192, 8192, 8192, name="extend-1x8k-prompt"),
        # the next chunk of two long prompts whose beginning stands in an 8-bit cache
        _case("extend", QWEN_7B, 2, 20000, 32768, 2048, 2048, name="extend-2x2k-chunk-8bit", kv8=True),
        # a server's mixed batch: a chunk of one prompt beside single tokens of the others
        _case("extend", QWEN_1_5B, 24, 500, 4000, 500, 1000, name="extend-mixed", singles=True, pad=5),
    ]


# What a drawn case may cost at most: bytes of the caches, and values of the plain form's scores
_MOST_BYTES = 1.6e9
_MOST_SCORES = 4.0e9


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["append", "append", "full", "sparse", "extend", "extend", "extend"])
        model = rng.choice(MODELS)
        kv8 = kind in ("full", "sparse") or rng.random() < 0.4
        batch = _log(rng, 1, 96)
        hi = _log(rng, 1 if kind in ("append", "extend") else 64, 100000)
        lo = hi if rng.random() < 0.3 else int(hi * rng.uniform(0.2, 0.95))
        new_hi, new_lo, singles = 1, 1, False
        if kind in ("append", "extend"):
            shape = rng.choice(["one", "few", "run", "prompt", "singles"])
            if shape == "few":
                new_lo, new_hi = rng.choice([0, 1]), min(hi, rng.randint(2, 16))
            elif shape in ("run", "singles"):
                new_hi = _log(rng, 1, hi)
                new_lo, singles = max(1, new_hi // 2), shape == "singles"
            elif shape == "prompt":
                new_lo, new_hi = lo, hi
            lo = max(lo, new_lo)
        else:
            lo = max(lo, 1)
        wide = 1 if kv8 else 2
        rows = (new_hi + batch - 1) if singles else batch * new_hi
        size = batch * hi * 2 * model["hkv"] * model["d"] * wide
        size += rows * 4 * model["hq"] * model["d"]
        scores = float(batch) * new_hi * model["hq"] * hi if kind == "extend" else 0.0
        if size > _MOST_BYTES or scores > _MOST_SCORES:
            continue
        return _case(kind, model, batch, lo, hi, new_lo, new_hi, singles=singles, kv8=kv8,
                     pad=rng.choice([0, 0, 3, 40]), packed=rng.random() < 0.6,
                     rot=rng.choice([model["d"], model["d"], model["d"] // 2]),
                     interleaved=rng.random() < 0.3, budget=PAGE * rng.choice([32, 64, 100, 128, 256]))


# ---- inputs ------------------------------------------------------------------------------

def _counts(case):
    """Tokens held and new tokens of every sequence: the case's own, whatever the seed, so that
    its outputs have one shape."""
    B = case["batch"]
    g = torch.Generator().manual_seed(31 * case["hi"] + 7 * case["lo"] + 1009 * B + case["new_hi"])
    lens = torch.randint(case["lo"], case["hi"] + 1, (B,), generator=g)
    lens[int(torch.randint(0, B, (1,), generator=g))] = case["hi"]
    new = torch.randint(case["new_lo"], case["new_hi"] + 1, (B,), generator=g)
    if case["singles"]:
        new[1:] = 1
    if case["new_lo"] == case["lo"] and case["new_hi"] == case["hi"] and not case["singles"]:
        new = lens.clone()
    return lens.tolist(), torch.minimum(new, lens).tolist()


def _values(shape, g):
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def _cache(case, n_pages, g, scale):
    """Keys or values of a cache that is already filled: normal values, a few tokens' larger."""
    x = torch.randn((n_pages, case["hkv"], PAGE, case["d"]), generator=g, device="cuda")
    x *= 1.0 + 2.0 * (torch.rand((n_pages, 1, PAGE, 1), generator=g, device="cuda") < 0.02)
    if not case["kv8"]:
        return x.to(torch.bfloat16)
    return x.div_(scale[:, None, None]).clamp_(-448, 448).to(torch.float8_e4m3fn)


def _selection(case, lens, g):
    """A sparse layer's selection, as a Delta layer leaves it: the last 8 pages and the best-scored
    older ones, ascending."""
    K = case["budget"] // PAGE
    idx = torch.full((case["batch"], K), -1, dtype=torch.int32)
    cnt = torch.empty((case["batch"],), dtype=torch.int32)
    for b, s in enumerate(lens):
        n = -(-s // PAGE)
        cnt[b] = min(n, K)
        keep = torch.arange(n)
        if n > K:
            old = torch.randperm(n - 8, generator=g)[:K - 8].sort().values
            keep = torch.cat([old, torch.arange(n - 8, n)])
        idx[b, :keep.numel()] = keep.int()
    return idx.cuda(), cnt.cuda()


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.Generator().manual_seed(seed * 7 + 3)
    B, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    lens, new = _counts(case)
    pages = [-(-s // PAGE) for s in lens]
    width, total = max(max(pages), 1), max(sum(pages), 1)
    pool = torch.randperm(total, generator=h).int()
    table = torch.zeros((B, width), dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = pool[at:at + n]
        at += n
    offsets = torch.zeros((B + 1,), dtype=torch.int32)
    offsets[1:] = torch.cumsum(torch.tensor(new), 0).int()
    scale = 0.02 + 0.04 * torch.rand((2, hkv), generator=g, device="cuda")
    x = dict(case=case, lens=lens, new=new, bound=max(max(lens), 1), max_new=max(new),
             page_table=table.cuda(), seq_lens=torch.tensor(lens, dtype=torch.int32).cuda(),
             row_offsets=offsets.cuda(), k_scale=scale[0].contiguous(), v_scale=scale[1].contiguous())
    rows = sum(new) + case["pad"]
    if case["kind"] == "append":
        kind = torch.float8_e4m3fn if case["kv8"] else torch.bfloat16
        x["k_cache"] = torch.zeros((total, hkv, PAGE, d), device="cuda").to(kind)
        x["v_cache"] = torch.zeros((total, hkv, PAGE, d), device="cuda").to(kind)
        if case["packed"]:
            qkv = _values((rows, hq + 2 * hkv, d), g)
            x["q"], x["k"], x["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        else:
            x["q"], x["k"], x["v"] = (_values((rows, n, d), g) for n in (hq, hkv, hkv))
        n = case["rot"] // 2
        x["inv_freq"] = (10000.0 ** (-torch.arange(n, dtype=torch.float64) / n)).float().cuda()
    else:
        x["k_cache"] = _cache(case, total, g, x["k_scale"])
        x["v_cache"] = _cache(case, total, g, x["v_scale"])
        x["q"] = _values((B if case["kind"] != "extend" else rows, hq, d), g)
    x["out"] = torch.zeros((x["q"].shape[0], hq, d), dtype=torch.bfloat16, device="cuda")
    if case["kind"] == "sparse":
        x["sel_idx"], x["sel_cnt"] = _selection(case, lens, h)
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    if own:
        from paper_2510_09883_amd import delta as D, extend as E
        shape = D.make_shape(case["batch"], case["hq"], case["hkv"], case["d"],
                             x["page_table"].shape[1], x["bound"])
        x["shape"] = shape
        scales = dict(k_scale=x["k_scale"], v_scale=x["v_scale"]) if case["kv8"] else {}
        x["kv"] = D.make_kv(x["k_cache"], x["v_cache"], x["page_table"], x["seq_lens"], **scales)
        if case["kind"] == "sparse":
            x["sel"] = D.make_select(case["budget"], 8 * PAGE)
        if case["kind"] in ("full", "sparse"):
            x["ws"] = D.alloc_workspace(shape, x.get("sel"))
        if case["kind"] == "extend":
            x["ws"] = E.alloc_extend_workspace(shape, x["q"].shape[0], x["max_new"])
    return x


def run(x):
    kind = x["case"]["kind"]
    if not own:
        return {"append": _plain_append, "full": _plain_decode, "sparse": _plain_decode,
                "extend": _plain_extend}[kind](x)
    from paper_2510_09883_amd import delta as D, extend as E
    if kind == "append":
        E.delta_rope_append(x["shape"], x["kv"], x["q"], x["k"], x["v"], x["out"], x["inv_freq"],
                            row_offsets=x["row_offsets"], interleaved=x["case"]["interleaved"])
        return {"q": x["out"], "k_cache": x["k_cache"], "v_cache": x["v_cache"]}
    if kind == "full":
        D.delta_full_attn(x["shape"], x["kv"], x["q"], x["out"], x["ws"])
    elif kind == "sparse":
        D.delta_sparse_attn(x["shape"], x["kv"], x["q"], x["out"], x["sel"], x["sel_idx"], x["sel_cnt"],
                            x["ws"])
    else:
        E.delta_extend_attn(x["shape"], x["kv"], x["q"], x["out"], x["row_offsets"], x["max_new"], x["ws"])
    return {"out": x["out"]}


# ---- the plain forms ---------------------------------------------------------------------

def _token_of_rows(x, rows):
    """Sequence and cache index of every row (past the last run: the last sequence, index 0),
    and which rows belong to a run."""
    r = torch.arange(rows, device="cuda")
    b = torch.searchsorted(x["row_offsets"].long(), r, right=True).sub_(1).clamp_(max=len(x["lens"]) - 1)
    real = r < x["row_offsets"][-1]
    t = x["seq_lens"].long()[b] - (x["row_offsets"].long()[b + 1] - r)
    return b, torch.where(real, t, 0), real


def _rotate(v, cos, sin, interleaved):
    n = cos.shape[-1]
    w = v.float()
    a, b = (w[..., 0:2 * n:2], w[..., 1:2 * n:2]) if interleaved else (w[..., :n], w[..., n:2 * n])
    lo, hi = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((lo, hi), -1).flatten(-2) if interleaved else torch.cat((lo, hi), -1)
    return torch.cat((turned, w[..., 2 * n:]), -1)


def _plain_append(x):
    """Rotation in 32 bits (the angles, up to 1e5 radians, in 64), rounded once to the cache's type."""
    case, total = x["case"], sum(x["new"])
    b, t, _ = _token_of_rows(x, total)
    angle = t.double()[:, None] * x["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x["out"][:total] = _rotate(x["q"][:total], cos, sin, case["interleaved"]).to(torch.bfloat16)
    k = _rotate(x["k"][:total], cos, sin, case["interleaved"])
    v = x["v"][:total].float()
    page, row = x["page_table"].long()[b, t // PAGE], t % PAGE
    if case["kv8"]:
        k = (k / x["k_scale"][:, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
        v = (v / x["v_scale"][:, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
        x["k_cache"].view(torch.uint8)[page, :, row] = k.view(torch.uint8)
        x["v_cache"].view(torch.uint8)[page, :, row] = v.view(torch.uint8)
    else:
        x["k_cache"][page, :, row] = k.to(torch.bfloat16)
        x["v_cache"][page, :, row] = v.to(torch.bfloat16)
    return {"q": x["out"], "k_cache": x["k_cache"], "v_cache": x["v_cache"]}


def _gathered(x, cache, scale, pages):
    """[batch, hkv, tokens, d] in 32 bits of the listed logical pages of every sequence."""
    phys = torch.gather(x["page_table"].long(), 1, pages)
    if cache.dtype == torch.bfloat16:
        c = cache[phys].float()
    else:
        c = cache.view(torch.uint8)[phys].view(torch.float8_e4m3fn).float() * scale[:, None, None]
    return c.transpose(1, 2).flatten(2, 3)


def _attend(q, k, v, seen):
    """q [batch, hkv, rows, d]; seen: which tokens a row sees. A row that sees none gets zeros."""
    s = q @ k.transpose(2, 3).contiguous() / math.sqrt(q.shape[-1])
    s = s.masked_fill_(~seen, -math.inf)
    top = s.amax(-1, keepdim=True).clamp_(min=-1e30)
    p = s.sub_(top).exp_()
    return (p @ v) / p.sum(-1, keepdim=True).clamp_(min=1e-30)


def _plain_decode(x):
    case = x["case"]
    B, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    if case["kind"] == "full":
        pages = torch.arange(x["page_table"].shape[1], device="cuda").expand(B, -1)
        live = pages >= 0
    else:
        pages = x["sel_idx"].long().clamp(min=0)
        live = torch.arange(pages.shape[1], device="cuda") < x["sel_cnt"][:, None]
    tokens = (pages[:, :, None] * PAGE + torch.arange(PAGE, device="cuda")).flatten(1)
    seen = (tokens < x["seq_lens"][:, None]) & live.repeat_interleave(PAGE, 1)
    k = _gathered(x, x["k_cache"], x["k_scale"], pages)
    v = _gathered(x, x["v_cache"], x["v_scale"], pages)
    o = _attend(x["q"].float().view(B, hkv, hq // hkv, d), k, v, seen[:, None, None])
    x["out"].copy_(o.reshape(B, hq, d))
    return {"out": x["out"]}


def _plain_extend(x):
    """Every run padded to the longest, all tokens of every sequence gathered."""
    case, total, n = x["case"], sum(x["new"]), x["max_new"]
    B, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    if total == 0:
        return {"out": x["out"]}
    b, t, _ = _token_of_rows(x, total)
    j = torch.arange(total, device="cuda") - x["row_offsets"].long()[b]
    q = torch.zeros((B, n, hkv, hq // hkv, d), device="cuda")
    q[b, j] = x["q"][:total].float().view(total, hkv, hq // hkv, d)
    last = torch.full((B, n), -1, device="cuda")
    last[b, j] = t
    width = x["page_table"].shape[1]
    pages = torch.arange(width, device="cuda").expand(B, -1)
    k = _gathered(x, x["k_cache"], x["k_scale"], pages)
    v = _gathered(x, x["v_cache"], x["v_scale"], pages)
    seen = torch.arange(width * PAGE, device="cuda") <= last[:, :, None]
    seen = seen[:, None, :, None].expand(B, 1, n, hq // hkv, width * PAGE).flatten(2, 3)
    o = _attend(q.transpose(1, 2).flatten(2, 3), k, v, seen)
    o = o.view(B, hkv, n, hq // hkv, d).transpose(1, 2)[b, j]
    x["out"][:total] = o.reshape(total, hq, d).to(torch.bfloat16)
    return {"out": x["out"]}


# ---- what a pass cannot do without -------------------------------------------------------

def work(case):
    """Every row in and out once, every attended key and value once per sequence; 4 operations per
    query head, head size and attended token."""
    B, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    wide = 1 if case["kv8"] else 2
    held, new = 0.5 * (case["lo"] + case["hi"]), 0.5 * (case["new_lo"] + case["new_hi"])
    rows = new + B - 1 if case["singles"] else B * new
    token = 2.0 * hkv * d * wide
    if case["kind"] == "append":
        size = rows * (4 * hq * d + 4 * hkv * d + token + 4.0 / PAGE) + 8 * B
        return {"bytes": size, "flops": rows * 3.0 * (hq + hkv) * case["rot"]}
    if case["kind"] == "extend":
        seen = rows * max(held - 0.5 * (new if not case["singles"] else 1), 0.0)
        if case["new_lo"] == case["lo"] and case["new_hi"] == case["hi"] and not case["singles"]:
            lo, hi = case["lo"], case["hi"]     # whole prompts: the mean of s * (s + 1) / 2
            seen = B * 0.5 * ((lo * lo + lo * hi + hi * hi) / 3.0 + held)
        return {"bytes": B * held * (token + 4.0 / PAGE) + rows * 4.0 * hq * d + 8 * B,
                "flops": 4.0 * hq * d * seen}
    if case["kind"] == "sparse":
        held = min(held, case["budget"])
    return {"bytes": B * (held * (token + 4.0 / PAGE) + 4.0 * hq * d + 4), "flops": 4.0 * B * hq * d * held}


# ---- the same results in 64 bits ---------------------------------------------------------

def _exact_rows(x, cache, scale, b, tokens):
    """float64 [n, hkv, d] of one sequence's tokens."""
    at = x["page_table"][b].long()[tokens // PAGE], slice(None), tokens % PAGE
    if cache.dtype == torch.bfloat16:
        return cache[at].double()
    return cache.view(torch.uint8)[at].view(torch.float8_e4m3fn).double() * scale.double()[:, None]


def _exact_append(x, case):
    out = x["out"].double()
    caches = [x["k_cache"].double(), x["v_cache"].double()]
    n, row = case["rot"] // 2, 0
    for b, (s, m) in enumerate(zip(x["lens"], x["new"])):
        t = torch.arange(s - m, s, device="cuda")
        rows = slice(row, row + m)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                           t.double()[:, None] * x["inv_freq"].double())[:, None]
        turned = []
        for w in (x["q"][rows].double(), x["k"][rows].double()):
            pair = (w[..., 0:2 * n:2], w[..., 1:2 * n:2]) if case["interleaved"] else (w[..., :n], w[..., n:2 * n])
            z = torch.complex(*pair) * turn
            w = w.clone()
            if case["interleaved"]:
                w[..., 0:2 * n:2], w[..., 1:2 * n:2] = z.real, z.imag
            else:
                w[..., :n], w[..., n:2 * n] = z.real, z.imag
            turned.append(w)
        out[rows] = turned[0]
        page = x["page_table"][b].long()[t // PAGE]
        for cache, w, scale in zip(caches, (turned[1], x["v"][rows].double()), (x["k_scale"], x["v_scale"])):
            if case["kv8"]:
                w = (w / scale.double()[:, None]).clamp(-448, 448)
            cache[page, :, t % PAGE] = w
        row += m
    return {"q": out, "k_cache": caches[0], "v_cache": caches[1]}


def exact(case, seed):
    x = _inputs(case, seed)
    if case["kind"] == "append":
        return _exact_append(x, case)
    hkv, G, d = case["hkv"], case["hq"] // case["hkv"], case["d"]
    out = torch.zeros(x["q"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for b, s in enumerate(x["lens"]):
        tokens = torch.arange(s, device="cuda")
        m, rows = 1, slice(b, b + 1)
        if case["kind"] == "extend":
            m, rows = x["new"][b], slice(row, row + x["new"][b])
            row += m
        if case["kind"] == "sparse":
            chosen = x["sel_idx"][b, :int(x["sel_cnt"][b])].long()
            tokens = (chosen[:, None] * PAGE + torch.arange(PAGE, device="cuda")).flatten()
            tokens = tokens[tokens < s]
        if m == 0:
            continue
        k = _exact_rows(x, x["k_cache"], x["k_scale"], b, tokens)
        v = _exact_rows(x, x["v_cache"], x["v_scale"], b, tokens)
        hidden = tokens[None] > torch.arange(s - m, s, device="cuda")[:, None]
        for h in range(hkv):
            q = x["q"][rows, h * G:(h + 1) * G].double()
            kh, vh = k[:, h].t().contiguous(), v[:, h].contiguous()
            for g in range(G):
                w = (q[:, g] @ kh / math.sqrt(d)).masked_fill_(hidden, -math.inf)
                out[rows, h * G + g] = torch.softmax(w, -1) @ vh
    return {"out": out}
