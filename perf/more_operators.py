"""Timed cases of the operators for a round of drafted tokens that form a tree, over the paged KV cache.

`kind` "append": `delta_norm_rope_append`, a norm of every head's queries and keys, their rotation and
the write to the cache.  "layout": `delta_tree_layout`, positions and visible rows of trees given by
parents.  "tree": `delta_tree_attn`, attention of every row to the cached tokens before its run and to
its ancestors.  "verify": `delta_verify_drafts`, which drafts the target's probabilities accept, and the
token after them.  "compact": `delta_cache_compact`, the accepted rows brought together in the caches of
all layers.

Plain values of a case: heads `hq`/`hkv`, head size `d`, `batch` sequences that hold `lo`..`hi` tokens
(drawn uniformly, one of them `hi`), of which `new_lo`..`new_hi` are new, `kv8` (e4m3 caches with one
scale per KV head, else bf16), `pad` rows behind the last run, `wide` (how many rows back a row's parent
may lie: 1 is a chain), `tree` (appended rows have their depths as positions), `rot` rotated values per
head, `interleaved` pairs, `f32` (norm weights in 32 bits), `vocab` tokens, `drafted` (the drafts'
probabilities are given, not only their tokens), `layers`.
"""
import math

import torch

own = False

PAGE = 16
EPS = 1e-6

# Head layouts of the models in paper_2510_09883_amd/configs.py (and rank shares of them)
LLAMA_8B = dict(hq=32, hkv=8, d=128)
QWEN_7B = dict(hq=28, hkv=4, d=128)
QWEN_14B = dict(hq=40, hkv=8, d=128)
QWEN_1_5B = dict(hq=12, hkv=2, d=128)
QWEN_14B_QUARTER = dict(hq=10, hkv=2, d=128)
SMALL = dict(hq=8, hkv=2, d=64)
MODELS = [LLAMA_8B, QWEN_7B, QWEN_14B, QWEN_1_5B, QWEN_14B_QUARTER, SMALL]
VOCAB = 151936   # of the decoder in bench.py


def _case(kind, model, batch, lo, hi, new_lo, new_hi, **kw):
    c = dict(kind=kind, **model, batch=batch, lo=lo, hi=hi, new_lo=new_lo, new_hi=new_hi, kv8=False, pad=0,
             wide=8, tree=True, rot=model["d"], interleaved=False, f32=False, vocab=VOCAB, drafted=False, layers=1)
    c.update(kw)
    return c


def listed():
    return [
        # one user's tree of drafts, where only latency counts
        _case("append", QWEN_7B, 1, 4096, 4096, 16, 16, name="append-1x16"),
        # a batch of prompts as a server collects them, padded behind the last one
        _case("append", LLAMA_8B, 4, 700, 2900, 700, 2900, name="append-4-prompts", tree=False, pad=37),
        # the trees of one user, and of a large batch
        _case("layout", QWEN_7B, 1, 1000, 4096, 16, 16, name="layout-1x16"),
        _case("layout", LLAMA_8B, 96, 300, 20000, 20, 64, name="layout-96x64", pad=11),
        # short ragged sequences of a small model, some with one row, some with none
        _case("tree", SMALL, 32, 3, 300, 0, 7, name="tree-32x7-short", pad=3),
        # one user's tree far into a decode
        _case("tree", QWEN_7B, 1, 8192, 8192, 16, 16, name="tree-1x16-8k"),
        # wide trees of a batch
        _case("tree", LLAMA_8B, 16, 4000, 16384, 64, 64, name="tree-16x64-16k"),
        # ragged trees over long 8-bit caches
        _case("tree", QWEN_14B, 12, 10000, 32768, 8, 24, name="tree-12x24-8bit", kv8=True),
        # one user's tree, drafted without sampling
        _case("verify", SMALL, 1, 300, 300, 16, 16, name="verify-1x16-tree"),
        # chains of a batch, drawn from the drafting model's probabilities
        _case("verify", SMALL, 64, 300, 300, 4, 8, name="verify-64x8-chains", wide=1, drafted=True),
        # one user's accepted drafts in every layer
        _case("compact", QWEN_7B, 1, 2000, 2000, 16, 16, name="compact-1x16", layers=28),
        # those of a batch
        _case("compact", QWEN_1_5B, 64, 100, 400, 6, 24, name="compact-64x24", layers=28),
    ]


# What a drawn case may cost at most (the largest listed one of its kind is larger): bytes of its
# inputs, and values of the plain form's scores
_MOST_BYTES = 0.65e9
_MOST_SCORES = 5.0e8


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["append", "append", "layout", "tree", "tree", "tree", "verify", "verify", "compact"])
        model = rng.choice(MODELS)
        kv8 = kind in ("append", "tree", "compact") and rng.random() < 0.4
        c = _case(kind, model, _log(rng, 1, 96), 1, 1, 1, 1, kv8=kv8, pad=rng.choice([0, 0, 3, 40]),
                  wide=rng.choice([1, 2, 8, 30]), rot=rng.choice([model["d"], model["d"], model["d"] // 2]),
                  interleaved=rng.random() < 0.3, f32=rng.random() < 0.3, drafted=rng.random() < 0.5)
        c["new_hi"] = _log(rng, 1, 256)
        c["new_lo"] = c["new_hi"] if rng.random() < 0.3 else int(c["new_hi"] * rng.uniform(0.0, 0.9))
        c["hi"] = c["new_hi"] + _log(rng, 1, 60000)
        c["lo"] = max(c["new_hi"], int(c["hi"] * rng.uniform(0.2, 1.0)))
        token = 2 * model["hkv"] * model["d"] * (1 if kv8 else 2)
        rows = c["batch"] * c["new_hi"]
        if kind == "append":
            if rng.random() < 0.4:   # prompts
                c["new_hi"], c["new_lo"], c["tree"] = c["hi"], c["lo"], False
                rows = c["batch"] * c["hi"]
            size = c["batch"] * c["hi"] * token + rows * 2 * model["d"] * (2 * model["hq"] + 2 * model["hkv"])
            if size > _MOST_BYTES / 2.5:
                continue
        elif kind == "layout":
            c["hi"] = c["new_hi"] + _log(rng, 1000, 60000)
            c["lo"] = max(c["new_hi"], c["hi"] // 3)
            if rows > 6000:
                continue
        elif kind == "tree":
            if c["batch"] * c["hi"] * token > _MOST_BYTES or rows * model["hq"] * c["hi"] > _MOST_SCORES:
                continue
        elif kind == "verify":
            c["vocab"] = rng.choice([_log(rng, 1000, 200000), VOCAB, 32000, 50257, 128256])
            if c["drafted"]:   # siblings that were drawn: a few
                c["wide"] = rng.choice([1, 1, 1, 2, 3])
            if rows * c["vocab"] * (8 if c["drafted"] else 4) > _MOST_BYTES:
                continue
        else:
            c["layers"] = rng.choice([1, 2, 28])
            c["new_lo"] = max(1, c["new_lo"])
            c["new_hi"] = max(c["new_hi"], c["new_lo"])
            if c["batch"] * c["hi"] * token * c["layers"] > _MOST_BYTES:
                continue
        return c


# ---- inputs ------------------------------------------------------------------------------

def _counts(case):
    """Tokens held and new tokens of every sequence: the case's own, whatever the seed, so that
    its outputs have one shape."""
    B = case["batch"]
    g = torch.Generator().manual_seed(31 * case["hi"] + 7 * case["lo"] + 1009 * B + case["new_hi"])
    lens = torch.randint(case["lo"], case["hi"] + 1, (B,), generator=g)
    lens[int(torch.randint(0, B, (1,), generator=g))] = case["hi"]
    new = torch.randint(case["new_lo"], case["new_hi"] + 1, (B,), generator=g)
    new[int(torch.randint(0, B, (1,), generator=g))] = case["new_hi"]
    if case["new_hi"] == case["hi"] and not case["tree"]:   # whole prompts
        new = lens.clone()
    return lens.tolist(), torch.minimum(new, lens).tolist()


def _parents(case, new, g):
    """Parents of every row, -1 for the first of a run; a row's parent is at most `wide` rows before it."""
    out = []
    for n in new:
        j = torch.arange(n)
        back = 1 + (torch.rand((n,), generator=g) * torch.clamp(j, max=case["wide"])).long()
        out.append(torch.where(j == 0, -1, j - torch.minimum(back, j.clamp(min=1))))
    return torch.cat(out + [torch.full((case["pad"],), -7)]).int()


def _ancestors(new, parents):
    """Depth of every row, and bool [rows, longest run]: which rows of its run it sees (host)."""
    sees = torch.zeros((len(parents), max(max(new), 1)), dtype=torch.bool)
    depth = torch.zeros((len(parents),), dtype=torch.int32)
    up, at = parents.tolist(), 0
    for n in new:
        for j in range(n):
            if up[at + j] >= 0:
                sees[at + j] = sees[at + up[at + j]]
                depth[at + j] = depth[at + up[at + j]] + 1
            sees[at + j, j] = True
        at += n
    return depth, sees


def _words(sees):
    """Bits of bool [rows, n] in int32 words, the lowest bit first."""
    rows, n = sees.shape
    words = -(-n // 32)
    bits = torch.zeros((rows, 32 * words), dtype=torch.int64, device=sees.device)
    bits[:, :n] = sees
    value = (bits.view(rows, words, 32) << torch.arange(32, device=sees.device)).sum(-1)
    return torch.where(value >= 2 ** 31, value - 2 ** 32, value).int()


def _values(shape, g):
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def _cache(case, n_pages, g, scale):
    """Keys or values of a cache that is already filled: normal values, a few tokens' larger."""
    x = torch.randn((n_pages, case["hkv"], PAGE, case["d"]), generator=g, device="cuda")
    x *= 1.0 + 2.0 * (torch.rand((n_pages, 1, PAGE, 1), generator=g, device="cuda") < 0.02)
    if not case["kv8"]:
        return x.to(torch.bfloat16)
    return x.div_(scale[:, None, None]).clamp_(-448, 448).to(torch.float8_e4m3fn)


def _pages(x, case, lens, h):
    """A shuffled page table."""
    pages = [-(-s // PAGE) for s in lens]
    width, total = max(max(pages), 1), max(sum(pages), 1)
    pool = torch.randperm(total, generator=h).int()
    table = torch.zeros((len(lens), width), dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = pool[at:at + n]
        at += n
    x["page_table"], x["pages"] = table.cuda(), total


def _probabilities(x, case, rows, parents, new, g, h):
    """Peaked distributions of the target and (`drafted`) of a drafting model that is near it, tokens
    that the latter drew or, without it, likely tokens of the target, and uniform numbers."""
    vocab = case["vocab"]
    logits = torch.randn((rows, vocab), generator=g, device="cuda").mul_(2.5)
    near = logits + 0.5 * torch.randn((rows, vocab), generator=g, device="cuda")
    x["target"] = torch.softmax(logits, -1)
    x["draft"] = torch.softmax(near, -1) if case["drafted"] else None
    x["uniform"] = torch.rand((rows,), generator=g, device="cuda")
    first = torch.tensor([0] + new).cumsum(0)[:-1]
    run = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new))
    parent = torch.zeros((rows,), dtype=torch.long)
    parent[:len(run)] = first[run] + parents[:len(run)].long().clamp(min=0)
    if case["drafted"]:
        noise = torch.rand((rows, vocab), generator=g, device="cuda").clamp_(min=1e-20)
        tokens = (x["draft"][parent.cuda()].clamp_(min=1e-30).log() - (-noise.log()).log()).argmax(-1)
    else:   # siblings have tokens of their own, the likeliest of a noisy guess
        rank, count = torch.zeros((rows,), dtype=torch.long), {}
        for r in range(len(run)):
            p = int(parent[r])
            rank[r] = count.get(p, 0)
            count[p] = int(rank[r]) + 1
        near.add_(torch.randn((rows, vocab), generator=g, device="cuda"))
        k = min(vocab, int(rank.max()) + 1)
        best = torch.topk(near, k, -1).indices
        tokens = best[parent.cuda(), rank.clamp(max=k - 1).cuda()]
    x["tokens"] = tokens.int()


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.Generator().manual_seed(seed * 7 + 3)
    B, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    lens, new = _counts(case)
    if case["kind"] == "layout":   # (its outputs' shape goes by the runs alone)
        lens = torch.randint(max(case["lo"], case["new_hi"]), case["hi"] + 1, (B,), generator=h).tolist()
    rows = sum(new) + case["pad"]
    offsets = torch.zeros((B + 1,), dtype=torch.int32)
    offsets[1:] = torch.cumsum(torch.tensor(new), 0).int()
    x = dict(case=case, lens=lens, new=new, bound=max(max(lens), 1), max_new=max(new), rows=rows,
             seq_lens=torch.tensor(lens, dtype=torch.int32).cuda(), row_offsets=offsets.cuda())
    kind = case["kind"]
    if kind in ("layout", "tree", "verify") or (kind == "append" and case["tree"]):
        parents = _parents(case, new, h)
        x["parents"] = parents.cuda()
    if kind == "verify":
        _probabilities(x, case, rows, parents, new, g, h)
        x["path"] = torch.zeros((B, max(x["max_new"], 1)), dtype=torch.int32, device="cuda")
        x["n_path"], x["next"] = (torch.zeros((B,), dtype=torch.int32, device="cuda") for _ in range(2))
        return x
    if kind == "layout":
        words = max(1, -(-x["max_new"] // 32))
        x["positions"] = torch.zeros((rows,), dtype=torch.int32, device="cuda")
        x["masks"] = torch.zeros((rows, words), dtype=torch.int32, device="cuda")
        return x
    _pages(x, case, lens, h)
    scale = 0.02 + 0.04 * torch.rand((2, hkv), generator=g, device="cuda")
    x["k_scale"], x["v_scale"] = scale[0].contiguous(), scale[1].contiguous()
    if kind == "compact":
        # accepted rows that lie behind those that they replace, as those of wide trees do
        x["path"] = torch.full((B, x["max_new"]), -1, dtype=torch.int32)
        x["n_path"] = torch.zeros((B,), dtype=torch.int32)
        for b, n in enumerate(new):
            c = int(torch.randint(1, min((n + 1) // 2, 8) + 1, (1,), generator=h))
            x["path"][b, 0], x["n_path"][b] = 0, c
            x["path"][b, 1:c] = (c + torch.randperm(n - c, generator=h)[:c - 1]).sort().values.int()
        x["path"], x["n_path"] = x["path"].cuda(), x["n_path"].cuda()
        x["caches"] = [(_cache(case, x["pages"], g, x["k_scale"]), _cache(case, x["pages"], g, x["v_scale"]))
                       for _ in range(case["layers"])]
        x["new_lens"] = torch.zeros((B,), dtype=torch.int32, device="cuda")
        return x
    if kind == "append":
        kept = torch.float8_e4m3fn if case["kv8"] else torch.bfloat16
        x["k_cache"] = torch.zeros((x["pages"], hkv, PAGE, d), device="cuda").to(kept)
        x["v_cache"] = torch.zeros((x["pages"], hkv, PAGE, d), device="cuda").to(kept)
        qkv = _values((rows, hq + 2 * hkv, d), g)
        x["q"], x["k"], x["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        weights = 1.0 + 0.2 * torch.randn((2, d), generator=g, device="cuda")
        weights = weights if case["f32"] else weights.to(torch.bfloat16)
        x["q_weight"], x["k_weight"] = weights[0].contiguous(), weights[1].contiguous()
        n = case["rot"] // 2
        x["inv_freq"] = (10000.0 ** (-torch.arange(n, dtype=torch.float64) / n)).float().cuda()
        x["positions"] = None
        if case["tree"]:
            before = torch.repeat_interleave(torch.tensor(lens) - torch.tensor(new), torch.tensor(new)).int()
            depth = _ancestors(new, parents)[0]
            depth[:len(before)] += before
            x["positions"] = depth.cuda()
    else:
        x["k_cache"] = _cache(case, x["pages"], g, x["k_scale"])
        x["v_cache"] = _cache(case, x["pages"], g, x["v_scale"])
        x["q"] = _values((rows, hq, d), g)
        x["sees"] = _ancestors(new, parents)[1]
        x["masks"] = _words(x["sees"]).cuda()
    x["out"] = torch.zeros((rows, hq, d), dtype=torch.bfloat16, device="cuda")
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    if not own:
        return x
    from paper_2510_09883_amd import delta as D, drafts as T
    kind = case["kind"]
    scales = dict(k_scale=x["k_scale"], v_scale=x["v_scale"]) if case["kv8"] else {}
    if kind == "verify":
        x["ws"] = T.alloc_verify_workspace(case["batch"], case["vocab"])
        return x
    width = x["page_table"].shape[1] if "page_table" in x else -(-x["bound"] // PAGE)
    x["shape"] = D.make_shape(case["batch"], case["hq"], case["hkv"], case["d"], width, x["bound"])
    if kind in ("append", "tree"):
        x["kv"] = D.make_kv(x["k_cache"], x["v_cache"], x["page_table"], x["seq_lens"], **scales)
    if kind == "tree":
        x["ws"] = T.alloc_tree_workspace(x["shape"], x["rows"], x["max_new"])
    if kind == "compact":
        x["stack"] = T.CacheStack(x["shape"], [D.make_kv(k, v, x["page_table"], x["seq_lens"], **scales)
                                               for k, v in x["caches"]])
    return x


def run(x):
    kind, case = x["case"]["kind"], x["case"]
    if not own:
        return {"append": _plain_append, "layout": _plain_layout, "tree": _plain_tree, "verify": _plain_verify,
                "compact": _plain_compact}[kind](x)
    from paper_2510_09883_amd import drafts as T
    if kind == "append":
        T.delta_norm_rope_append(x["shape"], x["kv"], x["q"], x["k"], x["v"], x["out"], x["q_weight"], x["k_weight"],
                                 EPS, x["inv_freq"], row_offsets=x["row_offsets"], positions=x["positions"],
                                 interleaved=case["interleaved"])
        return {"q": x["out"], "k_cache": x["k_cache"], "v_cache": x["v_cache"]}
    if kind == "layout":
        T.delta_tree_layout(x["shape"], x["seq_lens"], x["parents"], x["positions"], x["masks"], x["row_offsets"],
                            x["max_new"])
        return {"positions": x["positions"], "masks": x["masks"]}
    if kind == "tree":
        T.delta_tree_attn(x["shape"], x["kv"], x["q"], x["out"], x["masks"], x["row_offsets"], x["max_new"], x["ws"])
        return {"out": x["out"]}
    if kind == "verify":
        T.delta_verify_drafts(x["target"], x["draft"], x["tokens"], x["parents"], x["uniform"], x["row_offsets"],
                              x["path"], x["n_path"], x["next"], x["ws"])
        return {"path": x["path"], "n_path": x["n_path"], "next": x["next"]}
    T.delta_cache_compact(x["stack"], x["rows"], x["row_offsets"], x["path"], x["n_path"], x["new_lens"])
    return {"caches": x["caches"], "new_lens": x["new_lens"]}


# ---- the plain forms ---------------------------------------------------------------------

def _token_of_rows(x, rows):
    """Sequence, place in the run and token index of the first `rows` rows."""
    r = torch.arange(rows, device="cuda")
    b = torch.searchsorted(x["row_offsets"].long(), r, right=True).sub_(1).clamp_(max=len(x["lens"]) - 1)
    j = r - x["row_offsets"].long()[b]
    return b, j, x["seq_lens"].long()[b] - (x["row_offsets"].long()[b + 1] - r)


def _rotate(v, cos, sin, interleaved):
    n = cos.shape[-1]
    a, b = (v[..., 0:2 * n:2], v[..., 1:2 * n:2]) if interleaved else (v[..., :n], v[..., n:2 * n])
    lo, hi = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((lo, hi), -1).flatten(-2) if interleaved else torch.cat((lo, hi), -1)
    return torch.cat((turned, v[..., 2 * n:]), -1)


def _plain_append(x):
    """Norm and rotation in 32 bits (the angles, up to 1e5 radians, in 64), rounded once to the cache's type."""
    case, total = x["case"], sum(x["new"])
    b, _, t = _token_of_rows(x, total)
    p = t if x["positions"] is None else x["positions"][:total]
    angle = p.double()[:, None] * x["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(v, weight):
        v = v[:total].float()
        v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS) * weight.float()
        return _rotate(v, cos, sin, case["interleaved"])
    x["out"][:total] = turned(x["q"], x["q_weight"]).to(torch.bfloat16)
    k = turned(x["k"], x["k_weight"])
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


def _plain_layout(x):
    """Rows of all runs in the order of their place in the run: a parent's bits stand when it is needed."""
    total, n = sum(x["new"]), x["max_new"]
    b, j, t = _token_of_rows(x, total)
    B = len(x["lens"])
    up = torch.full((B, n + 1), -1, device="cuda")
    up[b, j] = x["parents"][:total].long()
    sees = torch.zeros((B, n + 1, max(n, 1)), dtype=torch.bool, device="cuda")   # (the last: no parent)
    depth = torch.full((B, n + 1), -1, device="cuda")
    seq = torch.arange(B, device="cuda")
    for i in range(n):
        p = torch.where(up[:, i] < 0, n, up[:, i])
        sees[:, i] = sees[seq, p]
        sees[:, i, i] = True
        depth[:, i] = depth[seq, p] + 1
    x["masks"][:total] = _words(sees[b, j])
    x["positions"][:total] = (t - j + depth[b, j]).int()
    return {"positions": x["positions"], "masks": x["masks"]}


def _gathered(x, cache, scale):
    """[batch, hkv, tokens, d] in 32 bits of all pages of every sequence."""
    phys = x["page_table"].long()
    if cache.dtype == torch.bfloat16:
        c = cache[phys].float()
    else:
        c = cache.view(torch.uint8)[phys].view(torch.float8_e4m3fn).float() * scale[:, None, None]
    return c.transpose(1, 2).flatten(2, 3)


def _plain_tree(x):
    """Every run padded to the longest, all tokens of every sequence gathered."""
    case, total, n = x["case"], sum(x["new"]), x["max_new"]
    B, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    if total == 0:
        return {"out": x["out"]}
    b, j, _ = _token_of_rows(x, total)
    q = torch.zeros((B, n, hkv, hq // hkv, d), device="cuda")
    q[b, j] = x["q"][:total].float().view(total, hkv, hq // hkv, d)
    k, v = _gathered(x, x["k_cache"], x["k_scale"]), _gathered(x, x["v_cache"], x["v_scale"])
    width = k.shape[2]
    bits = (x["masks"][:total, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
    rows = torch.zeros((B, n, bits.shape[1] * 32), dtype=torch.bool, device="cuda")
    rows[b, j] = bits.flatten(1).bool()
    before = x["seq_lens"].long() - (x["row_offsets"][1:] - x["row_offsets"][:-1]).long()
    place = torch.arange(width, device="cuda") - before[:, None]           # of a token in the run
    inside = (place >= 0) & (place < (x["seq_lens"].long() - before)[:, None])
    seen = torch.gather(rows, 2, place.clamp(0, rows.shape[2] - 1)[:, None].expand(B, n, width))
    seen = (seen & inside[:, None]) | (place < 0)[:, None]
    seen = seen[:, None, :, None].expand(B, 1, n, hq // hkv, width).flatten(2, 3)
    s = q.transpose(1, 2).flatten(2, 3) @ k.transpose(2, 3).contiguous() / math.sqrt(d)
    s = s.masked_fill_(~seen, -math.inf)
    top = s.amax(-1, keepdim=True).clamp_(min=-1e30)
    p = s.sub_(top).exp_()
    o = (p @ v) / p.sum(-1, keepdim=True).clamp_(min=1e-30)
    o = o.view(B, hkv, n, hq // hkv, d).transpose(1, 2)[b, j]
    x["out"][:total] = o.reshape(total, hq, d).to(torch.bfloat16)
    return {"out": x["out"]}


def _plain_verify(x):
    """All sequences step through the places of their runs together; sums and products in 64 bits."""
    case, B, n = x["case"], x["case"]["batch"], x["max_new"]
    off = x["row_offsets"].long()
    new = off[1:] - off[:-1]
    live = new > 0
    first = torch.where(live, off[:-1], 0)
    cur = torch.zeros((B,), dtype=torch.long, device="cuda")
    left = torch.ones((B,), dtype=torch.float64, device="cuda")
    r = x["target"][first].double()
    count = live.long()
    x["path"].fill_(-1)
    x["path"][:, 0] = torch.where(live, 0, -1).int()
    seq = torch.arange(B, device="cuda")
    for j in range(1, n):
        row = torch.where(j < new, first + j, first)
        tested = (j < new) & (x["parents"].long()[row] == cur)
        token = x["tokens"].long()[row]
        at = r[seq, token]
        chance = 1.0 if x["draft"] is None else x["draft"][first + cur, token].double()
        take = tested & (x["uniform"][row].double() * chance * left < at)
        drop = tested & ~take
        if x["draft"] is None:
            r[seq, token] = torch.where(drop, 0.0, at)
            left = torch.where(drop, left - at, left)
        else:
            rest = (r - left[:, None] * x["draft"][first + cur].double()).clamp_(min=0)
            r = torch.where(drop[:, None], rest, r)
            left = torch.where(drop, rest.sum(-1), left)
        cur = torch.where(take, j, cur)
        r = torch.where(take[:, None], x["target"][row].double(), r)
        left = torch.where(take, 1.0, left)
        x["path"][seq, torch.where(take, count, 0)] = torch.where(take, j, x["path"][:, 0].long()).int()
        count += take
    total = r.sum(-1)
    r = torch.where((total > 0)[:, None], r, x["target"][first + cur].double())
    c = torch.cumsum(r, -1)
    goal = x["uniform"][first].double() * c[:, -1]
    after = (c <= goal[:, None]).sum(-1)
    last = case["vocab"] - 1 - (r > 0).flip(-1).long().argmax(-1)
    token = torch.where(c[:, -1] > 0, torch.minimum(after, last), -1)
    x["next"].copy_(torch.where(live, token, -1))
    x["n_path"].copy_(count)
    return {"path": x["path"], "n_path": x["n_path"], "next": x["next"]}


def _plain_compact(x):
    new = x["row_offsets"].long()[1:] - x["row_offsets"].long()[:-1]
    before = x["seq_lens"].long() - new
    i = torch.arange(x["path"].shape[1], device="cuda")
    b, i = torch.nonzero(i[None] < x["n_path"][:, None], as_tuple=True)
    src, dst = before[b] + x["path"].long()[b, i], before[b] + i
    table = x["page_table"].long()
    for layer in x["caches"]:
        for cache in layer:
            c = cache.view(torch.uint8) if x["case"]["kv8"] else cache
            c[table[b, dst // PAGE], :, dst % PAGE] = c[table[b, src // PAGE], :, src % PAGE]
    x["new_lens"].copy_(before + x["n_path"])
    return {"caches": x["caches"], "new_lens": x["new_lens"]}


# ---- what a pass cannot do without -------------------------------------------------------

def work(case):
    """Every row in and out once, every cached key and value once per sequence; 4 operations per query
    head, head size and seen token; one row of probabilities per sequence, of the drafts' where given
    a second; every moved token in and out once."""
    B, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    lens, new = _counts(case)
    rows = sum(new)
    token = 2.0 * hkv * d * (1 if case["kv8"] else 2)
    if case["kind"] == "append":
        return {"bytes": rows * (4 * hq * d + 4 * hkv * d + token + 4.0 / PAGE) + 8 * B,
                "flops": rows * (hq + hkv) * (4.0 * d + 3.0 * case["rot"])}
    if case["kind"] == "layout":
        words = max(1, -(-max(new) // 32))
        return {"bytes": rows * (8.0 + 4 * words) + 8 * B, "flops": 1.0 * rows * words}
    if case["kind"] == "tree":
        seen = sum(n * (s - n) + n for s, n in zip(lens, new))
        return {"bytes": sum(s for s, n in zip(lens, new) if n) * (token + 4.0 / PAGE) + rows * 4.0 * hq * d + 8 * B,
                "flops": 4.0 * hq * d * seen}
    if case["kind"] == "verify":
        some = sum(1 for n in new if n)
        wide = 2 if case["drafted"] and rows > some else 1
        return {"bytes": some * wide * 4.0 * case["vocab"] + 12.0 * rows, "flops": some * wide * 2.0 * case["vocab"]}
    moved = sum(0.5 * (min((n + 1) // 2, 8) - 1) for n in new)   # (of 1 .. that many accepted rows, less the first)
    return {"bytes": case["layers"] * moved * 2 * token + 16 * B, "flops": 0.0}


# ---- the same results in 64 bits ---------------------------------------------------------

def _exact_append(x, case):
    out = x["out"].double()
    caches = [x["k_cache"].double(), x["v_cache"].double()]
    n, row = case["rot"] // 2, 0
    for b, (s, m) in enumerate(zip(x["lens"], x["new"])):
        t = torch.arange(s - m, s, device="cuda")
        rows = slice(row, row + m)
        p = t if x["positions"] is None else x["positions"][rows]
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                           p.double()[:, None] * x["inv_freq"].double())[:, None]
        turned = []
        for w, weight in ((x["q"][rows].double(), x["q_weight"]), (x["k"][rows].double(), x["k_weight"])):
            w = weight.double() * w * (w.square().sum(-1, keepdim=True) / case["d"] + EPS).rsqrt()
            pair = (w[..., 0:2 * n:2], w[..., 1:2 * n:2]) if case["interleaved"] else (w[..., :n], w[..., n:2 * n])
            z = torch.complex(*(y.contiguous() for y in pair)) * turn
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


def _exact_layout(x):
    """Each row's way to the root, one by one."""
    rows, words = x["masks"].shape
    masks, positions = [[0] * words for _ in range(rows)], [0] * rows
    up, at = x["parents"].tolist(), 0
    for s, n in zip(x["lens"], x["new"]):
        for j in range(n):
            i, depth = j, -1
            while i >= 0:
                masks[at + j][i // 32] |= 1 << (i % 32)
                i, depth = up[at + i], depth + 1
            positions[at + j] = s - n + depth
        at += n
    signed = [[w - (1 << 32) if w >> 31 else w for w in row] for row in masks]
    return {"positions": torch.tensor(positions, dtype=torch.int32).cuda(),
            "masks": torch.tensor(signed, dtype=torch.int32).view(rows, words).cuda()}


def _exact_tree(x, case):
    hkv, G, d = case["hkv"], case["hq"] // case["hkv"], case["d"]
    out = torch.zeros(x["q"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for b, (s, m) in enumerate(zip(x["lens"], x["new"])):
        rows = slice(row, row + m)
        row += m
        if m == 0:
            continue
        t = torch.arange(s, device="cuda")
        at = x["page_table"][b].long()[t // PAGE], slice(None), t % PAGE
        kv = []
        for cache, scale in ((x["k_cache"], x["k_scale"]), (x["v_cache"], x["v_scale"])):
            if case["kv8"]:
                kv.append(cache.view(torch.uint8)[at].view(torch.float8_e4m3fn).double() * scale.double()[:, None])
            else:
                kv.append(cache[at].double())
        hidden = torch.zeros((m, s), dtype=torch.bool, device="cuda")
        hidden[:, s - m:] = ~x["sees"][rows, :m].cuda()
        for h in range(hkv):
            q = x["q"][rows, h * G:(h + 1) * G].double()
            kh, vh = kv[0][:, h].t().contiguous(), kv[1][:, h].contiguous()
            for i in range(G):
                w = (q[:, i] @ kh / math.sqrt(d)).masked_fill_(hidden, -math.inf)
                out[rows, h * G + i] = torch.softmax(w, -1) @ vh
    return {"out": out}


def _exact_verify(x, case):
    """Sequence by sequence, children by children."""
    B, width = x["path"].shape
    paths, counts, tokens = torch.full((B, width), -1, dtype=torch.int32), [], []
    up, token, u = x["parents"].tolist(), x["tokens"].tolist(), x["uniform"].double().tolist()
    at = 0
    for b, n in enumerate(x["new"]):
        path, node = ([0] if n else []), 0
        r = x["target"][at].double() if n else None
        while n:
            mass, taken = 1.0, None
            for child in (j for j in range(node + 1, n) if up[at + j] == node):
                v = token[at + child]
                have = float(r[v])
                if x["draft"] is None:
                    if u[at + child] * mass < have:
                        taken = child
                        break
                    r[v] = 0.0
                    mass -= have
                else:
                    q = x["draft"][at + node].double()
                    if u[at + child] * float(q[v]) * mass < have:
                        taken = child
                        break
                    r = torch.relu(r - mass * q)
                    mass = float(r.sum())
            if taken is None:
                break
            node = taken
            path.append(node)
            r = x["target"][at + node].double()
        if n:
            if float(r.sum()) <= 0:
                r = x["target"][at + node].double()
            c = r.cumsum(0)
            goal = u[at] * c[-1]
            over = torch.nonzero(c > goal).flatten()
            some = torch.nonzero(r > 0).flatten()
            tokens.append(int(over[0] if len(over) else some[-1]) if len(some) else -1)
        else:
            tokens.append(-1)
        paths[b, :len(path)] = torch.tensor(path, dtype=torch.int32)
        counts.append(len(path))
        at += n
    return {"path": paths.cuda(), "n_path": torch.tensor(counts, dtype=torch.int32).cuda(),
            "next": torch.tensor(tokens, dtype=torch.int32).cuda()}


def _exact_compact(x):
    caches = [tuple(c.double() for c in layer) for layer in x["caches"]]
    lens = []
    for b, (s, n) in enumerate(zip(x["lens"], x["new"])):
        keep = x["path"][b, :int(x["n_path"][b])].tolist()
        lens.append(s - n + len(keep))
        for to, row in enumerate(keep):
            if row == to:
                continue
            (p0, r0), (p1, r1) = divmod(s - n + row, PAGE), divmod(s - n + to, PAGE)
            p0, p1 = int(x["page_table"][b, p0]), int(x["page_table"][b, p1])
            for layer in caches:
                for c in layer:
                    c[p1, :, r1] = c[p0, :, r0]
    return {"caches": caches, "new_lens": torch.tensor(lens, dtype=torch.int32).cuda()}


def exact(case, seed):
    x = _inputs(case, seed)
    kind = case["kind"]
    if kind == "append":
        return _exact_append(x, case)
    if kind == "layout":
        return _exact_layout(x)
    if kind == "tree":
        return _exact_tree(x, case)
    if kind == "verify":
        return _exact_verify(x, case)
    return _exact_compact(x)
