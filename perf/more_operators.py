"""What a serving loop does with a paged key/value cache beside appending and attending, as a list of cases to measure.

Drafts that are trees: `moe_tree_masks` turns parents into ancestor masks and positions, `moe_tree_attention` verifies them over the
cache.  A cache that may not grow: `moe_kv_weights` adds up the attention weight that every cached token receives, `moe_kv_select`
chooses what to keep.  Both end in `moe_kv_compact`, which moves what is kept to the front of its sequence.  A case is one call;
`run` is either the framework's call (`own`) or the same in elementary torch operations in fp32.

The batch sizes are those of the repository's workloads: 1 to 256 sequences, chunks of 512 tokens, prompts of up to 8192; the heads are
generic (groups of 1 to 16 query heads to a key/value head, 64 to 128 wide, 256 in a few draws).
"""
import math

import torch

own = False

DEV = "cuda:0"

# What a case may leave out.  D sequences of rows_lo to `rows` new tokens each, with kv_lo to kv_hi tokens in the cache (spread over the
# logarithm), then `prompts` sequences of P / 2 to P new tokens (P for a single one) behind `past` cached tokens.
# fmt: "" (the cache holds dtype) or "fp8".  words: mask words of a row, of 64 bits each.  per_head: every head keeps tokens of its own.
DEFAULTS = {"heads": 32, "kv_heads": 4, "dim": 128, "page": 16, "dtype": "bf16", "fmt": "", "D": 0, "rows": 1, "rows_lo": 0,
            "kv_lo": 1, "kv_hi": 1, "prompts": 0, "P": 0, "past": 0, "window": 0, "sinks": False, "lse": False, "words": 1,
            "decay": 1.0, "budget": 0, "first": 0, "recent": 0, "per_head": True}

WIDE = {"heads": 32, "kv_heads": 4, "dim": 128}      # eight query heads to a key/value head
HALF = {"heads": 64, "kv_heads": 8, "dim": 64}       # the same groups, half as wide
QUAD = {"heads": 32, "kv_heads": 8, "dim": 128}      # groups of four
FP8_MAX, MIN_EXP, BAD_EXP = 448.0, -100, 255


def listed():
    return [
        # a decode step's drafts: 16 trees of 8 tokens, nothing but latency
        {"name": "masks_step", "op": "masks", "D": 16, "rows": 8, "kv_lo": 64, "kv_hi": 1024},
        # the largest decode batch with large ragged trees, windowed, beside a chunk that is no tree
        {"name": "masks_large", "op": "masks", "D": 256, "rows_lo": 33, "rows": 200, "kv_lo": 300, "kv_hi": 4096, "words": 4,
         "window": 128, "prompts": 1, "P": 512, "past": 1024},
        # one user's draft early in a reply: launches and latency
        {"name": "tree_one", "op": "tree", **WIDE, "D": 1, "rows": 26, "kv_lo": 700, "kv_hi": 700},
        # drafts of up to 64 tokens over ragged histories: each key serves up to 256 rows of its group
        {"name": "tree_batch", "op": "tree", **QUAD, "D": 32, "rows_lo": 16, "rows": 64, "kv_lo": 512, "kv_hi": 8192},
        # a windowed layer with sinks over a quantised cache: small trees beside a prompt's chunk of 512 tokens
        {"name": "tree_window_fp8", "op": "tree", **HALF, "page": 32, "fmt": "fp8", "D": 64, "rows": 12, "kv_lo": 100, "kv_hi": 4096,
         "window": 128, "sinks": True, "lse": True, "prompts": 1, "P": 512, "past": 1536},
        # a decode step adds its rows' weights: streams the keys
        {"name": "weights_decode", "op": "weights", **WIDE, "D": 64, "kv_lo": 512, "kv_hi": 8192},
        # layered prefill: the weights of a whole 8192-token prompt
        {"name": "weights_prompt", "op": "weights", **WIDE, "prompts": 1, "P": 8192, "decay": 0.0},
        # long prompts judged by their last 32 tokens alone, over a quantised cache
        {"name": "weights_last_fp8", "op": "weights", **HALF, "page": 32, "fmt": "fp8", "D": 12, "rows": 32, "kv_lo": 1024,
         "kv_hi": 16384, "decay": 0.0},
        # a decode batch whose ragged sequences are to fit 1024 tokens
        {"name": "select_step", "op": "select", **QUAD, "D": 32, "kv_lo": 500, "kv_hi": 4096, "budget": 1024, "first": 4, "recent": 64},
        # two long prompts, cut to a sixteenth
        {"name": "select_long", "op": "select", **WIDE, "page": 64, "D": 2, "kv_lo": 131072, "kv_hi": 131072, "budget": 8192, "first": 4,
         "recent": 256},
        # 32 verified drafts of 16 tokens: the accepted paths move up, the same tokens for all heads
        {"name": "compact_accept", "op": "accept", **WIDE, "D": 32, "rows": 16, "kv_lo": 512, "kv_hi": 4096, "per_head": False},
        # 16 histories of 8192 tokens lose half of them, every head its own; the weights move along
        {"name": "compact_half", "op": "compact", **QUAD, "D": 16, "kv_lo": 8192, "kv_hi": 8192, "budget": 4096, "first": 4, "recent": 256},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges above; it costs no more than the largest listed one."""
    kind = rng.choice(["masks", "tree", "tree", "tree", "tree_window", "step", "step", "prompt", "last", "last", "select", "select",
                       "accept", "compact", "compact"])
    kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8, 16])
    c = {"heads": kv_heads * group, "kv_heads": kv_heads, "dim": rng.choice([64, 64, 80, 96, 112, 128, 128, 128, 256]),
         "page": rng.choice([8, 16, 16, 32, 64, 128]), "fmt": rng.choice(["", "fp8"]), "dtype": rng.choice(["bf16"] * 5 + ["f32"])}
    wide = c["dtype"] == "f32"
    if kind == "masks":
        words = rng.choice([1, 1, 2, 4])
        c.update(op="masks", D=_log_int(rng, 1, 256), rows=rng.randint(2, 64 * words), words=words, kv_lo=64 * words, kv_hi=4000,
                 window=rng.choice([0, 0, 3, 128]), prompts=rng.choice([0, 0, 1]), P=rng.randint(300, 2000))
        c["rows_lo"] = rng.randint(1, c["rows"])
    elif kind in ("tree", "tree_window"):
        words = rng.choice([1, 1, 1, 2])
        c.update(op="tree", D=_log_int(rng, 1, 16 if wide else 64), rows=rng.randint(2, 64 * words), words=words, kv_lo=rng.randint(1, 200),
                 kv_hi=_log_int(rng, 200, 2000 if wide else 8192), lse=rng.random() < 0.3, sinks=rng.random() < 0.2)
        c["rows_lo"] = rng.randint(1, c["rows"])
        if kind == "tree_window":
            c.update(window=_log_int(rng, 8, 1024), prompts=rng.choice([0, 0, 1]), P=rng.randint(130, 700), past=rng.randint(0, 900))
    elif kind == "step":
        c.update(op="weights", D=_log_int(rng, 1, 128), rows=rng.choice([1, 1, 1, 2, 4]), kv_lo=rng.randint(4, 64), kv_hi=_log_int(rng, 64, 8192),
                 decay=rng.choice([1.0, 1.0, 0.99]), window=rng.choice([0, 0, 0, 200]))
    elif kind == "prompt":
        c.update(op="weights", D=rng.randint(0, 16), kv_lo=16, kv_hi=1000, prompts=rng.choice([1, 1, 2]), P=_log_int(rng, 40, 800 if wide else 4000),
                 past=rng.choice([0, 0, rng.randint(1, 3000)]), decay=rng.choice([1.0, 0.0]))
    elif kind == "last":
        c.update(op="weights", D=_log_int(rng, 1, 16), rows=rng.randint(5, 70), kv_lo=rng.randint(70, 500),
                 kv_hi=_log_int(rng, 500, 3000 if wide else 16000), decay=0.0)
    elif kind == "select":
        hi = _log_int(rng, 64, 60000)
        c.update(op="select", D=_log_int(rng, 1, max(1, min(128, 400000 // hi))), kv_lo=rng.randint(1, 64), kv_hi=hi,
                 budget=_log_int(rng, 16, max(17, hi // 2)), first=rng.randint(0, 4), recent=rng.randint(0, 12))
    elif kind == "accept":
        c.update(op="accept", D=_log_int(rng, 1, 128), rows=rng.randint(2, 64), kv_lo=rng.randint(64, 300), kv_hi=_log_int(rng, 300, 4096),
                 per_head=False)
    else:
        hi = _log_int(rng, 100, 16000)
        c.update(op="compact", D=_log_int(rng, 1, max(1, min(64, 120000 // hi))), kv_lo=rng.randint(16, 100), kv_hi=hi,
                 budget=rng.randint(hi // 8, hi), first=rng.randint(0, 4), recent=rng.randint(0, 8))
    return c


def _full(case):
    return {**DEFAULTS, **case}


def _spread(i):
    return (i + 1) * 0.6180339887498949 % 1.0


def _lens(c):
    """(new rows, tokens in the cache with them) of every sequence."""
    rows, kv = [], []
    lo = c["rows_lo"] or c["rows"]
    for i in range(c["D"]):
        rows.append(lo + int((c["rows"] - lo + 1) * _spread(i + 3) * 0.999))
        kv.append(max(int(round(c["kv_lo"] * (c["kv_hi"] / c["kv_lo"]) ** _spread(i))), rows[-1]))
    for i in range(c["prompts"]):
        n = c["P"] if c["prompts"] == 1 else max(1, int(c["P"] * (0.5 + 0.5 * _spread(i))))
        rows.append(n)
        kv.append(c["past"] + n)
    return rows, kv


def _is_tree(c, n):
    return c["op"] in ("masks", "tree") and n <= 64 * c["words"]


def work(case):
    c = _full(case)
    rows, kv = _lens(c)
    T, Hq, Hk, D = sum(rows), c["heads"], c["kv_heads"], c["dim"]
    esz = 4 if c["dtype"] == "f32" else 2
    row = Hk * ((D + 1.0) if c["fmt"] == "fp8" else D * esz)            # keys (or values) of a cached token
    if c["op"] == "masks":
        return {"bytes": T * (8.0 + 8 * c["words"]), "flops": 0}
    if c["op"] == "select":
        kept = sum(min(k, c["budget"]) for k in kv)
        return {"bytes": 4.0 * Hk * (sum(k for k in kv if k > c["budget"]) + kept), "flops": 0}
    if c["op"] == "accept":
        return {"bytes": sum(_accepted(n) for n in rows) * (4.0 + 4.0 * row), "flops": 0}
    if c["op"] == "compact":
        kept = sum(min(k, c["budget"]) - min(c["first"], k) for k in kv if k > c["budget"])
        return {"bytes": kept * (4.0 * row + 12.0 * Hk) + 1.0, "flops": 0}
    pairs = seen = 0.0
    for n, k in zip(rows, kv):
        past, w = k - n, c["window"] or k
        if _is_tree(c, n):
            deep = 2.0 * math.log(n) + 1.0                             # tokens of a row's path, about
            pairs += n * (min(past, w) + deep)
        else:
            full = max(0, min(n, w - past))                            # rows whose window reaches back to position 0
            pairs += full * past + full * (full + 1) // 2 + (n - full) * w
        seen += min(k, n + w - 1)
    if c["op"] == "tree":
        nbytes = T * (2.0 * Hq * D * esz + 8.0 * c["words"] + (4.0 * Hq if c["lse"] else 0.0)) + 2.0 * seen * row
        return {"bytes": nbytes, "flops": 4.0 * Hq * D * pairs}
    held = sum(kv)
    return {"bytes": T * Hq * (D * esz + 4.0) + seen * row + held * Hk * (4.0 if c["decay"] == 0.0 else 8.0), "flops": 2.0 * Hq * D * pairs}


def _accepted(n):
    """Rows of a draft of n that are kept, about: a path's share."""
    return max(1, int(math.log2(n)))


def _quantised(x):
    """FP8 codes and scale bytes of rows x [..., dim] (fp32): the scale 2^e is the smallest power of two, e >= -100, that
    keeps the row within the codes' range."""
    amax = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=MIN_EXP)
    return torch.ldexp(x, -e).to(torch.float8_e4m3fn), (e + 127).squeeze(-1).to(torch.uint8)


def prepare(case, seed):
    """A cache with its page table, the batch's lengths, and what the call takes beside them."""
    c = _full(case)
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    rows, kv = _lens(c)
    S, T, ps, Hq, Hk, D = len(rows), sum(rows), c["page"], c["heads"], c["kv_heads"], c["dim"]
    need = [-(-k // ps) for k in kv]
    max_pages, n_pages = max(need) + 1, sum(need) + 7

    # pages are handed out in random order; entries that no token needs are -1
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    counts = torch.tensor(need, device=DEV)
    first = torch.cumsum(counts, 0) - counts
    at = torch.arange(max_pages, device=DEV)
    table = torch.where(at < counts[:, None], order[(first[:, None] + at).clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous()
    offsets = [0]
    for n in rows:
        offsets.append(offsets[-1] + n)
    st = {"case": c, "rows": rows, "kv": kv, "page_table": table, "row_offsets": torch.tensor(offsets, dtype=torch.int32, device=DEV),
          "kv_lens": torch.tensor(kv, dtype=torch.int32, device=DEV)}

    loud = torch.exp(0.5 * torch.randn(Hk, 1, D, generator=g, device=DEV))       # some channels of the keys are louder than others
    if c["op"] in ("tree", "weights", "accept", "compact"):
        def pages(channel):
            x = torch.randn(n_pages, Hk, ps, D, generator=g, device=DEV) * channel
            return _quantised(x.to(dt).float()) if c["fmt"] == "fp8" else (x.to(dt), None)

        st["k_pages"], st["k_scales"] = pages(loud)
        st["v_pages"], st["v_scales"] = pages(1.0)
    if c["op"] in ("tree", "weights"):        # queries as a view of a fused projection
        st["q"] = torch.randn(T, (Hq + 2 * Hk) * D, generator=g, device=DEV).to(dt)[:, :Hq * D].unflatten(1, (Hq, D))
    if c["op"] in ("masks", "tree"):
        # a row's parent is one of those before it, a later one more likely; a chunk's rows are a chain
        off, i = st["row_offsets"].long(), torch.arange(T, device=DEV)
        seq = torch.searchsorted(off[1:], i, right=True)
        i = i - off[seq]
        parent = (i * (0.3 + 0.7 * torch.rand(T, generator=g, device=DEV))).long()
        tree = (off[1:] - off[:-1] <= 64 * c["words"])[seq]
        st["parents"] = torch.where(i == 0, -1, torch.where(tree, torch.minimum(parent, i - 1), i - 1)).to(torch.int32)
    if c["op"] == "tree":
        st["masks"], st["positions"] = _plain_masks(st)
        st["sinks"] = torch.randn(Hq, generator=g, device=DEV) if c["sinks"] else None
        st["out"] = torch.empty(T, Hq, D, dtype=dt, device=DEV)
        st["lse"] = torch.empty(T, Hq, device=DEV) if c["lse"] else None
    if c["op"] in ("weights", "select", "accept", "compact"):
        # accumulated weights are positive, a few tokens have most of them, some (nearly) none
        w = torch.exp(1.5 * torch.randn(n_pages, Hk, ps, generator=g, device=DEV))
        st["scores"] = torch.where(torch.rand(n_pages, Hk, ps, generator=g, device=DEV) < 0.05, 0.0, w) if c["op"] != "accept" else None
    if c["op"] == "weights":
        # what attention leaves in a row's log-sum-exp, nearly: with keys like these its scores are normal, of this variance
        var = torch.matmul(st["q"].float().square().view(T, Hk, Hq // Hk, D).transpose(0, 1).reshape(Hk, -1, D),
                           loud.square().view(Hk, D, 1)).view(Hk, T, Hq // Hk).transpose(0, 1).reshape(T, Hq) / D
        off, i = st["row_offsets"].long(), torch.arange(T, device=DEV)
        seq = torch.searchsorted(off[1:], i, right=True)
        sees = st["kv_lens"].long()[seq] - off[seq + 1] + i + 1
        sees = sees.clamp(max=c["window"]) if c["window"] > 0 else sees
        st["lse"] = (torch.log(sees.float())[:, None] + 0.5 * var).contiguous()
    if c["op"] == "compact":
        keep = torch.full((S, Hk, c["budget"]), -1, dtype=torch.int32, device=DEV)
        for s, k in enumerate(kv):
            m = min(k, c["budget"])
            r = torch.rand(Hk, k, generator=g, device=DEV)
            r[:, :c["first"]] = 2.0
            r[:, k - c["recent"]:] = 2.0
            keep[s, :, :m] = r.topk(m, dim=1).indices.sort(dim=1).values.to(torch.int32)
        st["keep"] = keep
        st["keep_lens"] = st["kv_lens"].clamp(max=c["budget"])
        st["first"] = None
    if c["op"] == "accept":
        most = max(_accepted(n) for n in rows)
        r = torch.rand(S, max(rows), generator=g, device=DEV)
        r[:, 0] = 2.0                                                   # the first row is the token that was accepted before
        lens = torch.tensor([_accepted(n) for n in rows], device=DEV)
        n = torch.tensor(rows, device=DEV)
        at = torch.arange(max(rows), device=DEV)
        r = torch.where(at < n[:, None], r, -1.0)
        path = r.topk(most, dim=1).indices
        path = torch.where(torch.arange(most, device=DEV) < lens[:, None], path, 1 << 30).sort(dim=1).values
        st["first"] = (st["kv_lens"].long() - n).to(torch.int32)
        st["keep"] = torch.where(path < 1 << 30, path + st["first"].long()[:, None], -1).to(torch.int32)
        st["keep_lens"] = lens.to(torch.int32)
    return st


def run(state):
    c = state["case"]
    if own:
        return _run_own(state)
    if c["op"] == "masks":
        return list(_plain_masks(state))
    if c["op"] == "select":
        return _plain_select(state)
    if c["op"] in ("accept", "compact"):
        return _plain_compact(state)
    if c["op"] == "weights":
        if c["D"]:
            _plain_weights(state, 0, c["D"])
        if c["prompts"]:
            _plain_weights(state, c["D"], c["D"] + c["prompts"])
        return [state["scores"]]
    T = sum(state["rows"])
    out = torch.empty(T, c["heads"], c["dim"], device=DEV)
    lse = torch.empty(T, c["heads"], device=DEV)
    # the drafts and the prompts have lengths of their own: each padded to its longest
    if c["D"]:
        _plain_attention(state, 0, c["D"], out, lse)
    if c["prompts"]:
        _plain_attention(state, c["D"], c["D"] + c["prompts"], out, lse)
    out = out.to(state["q"].dtype)
    return [out, lse] if c["lse"] else [out]


def _cache(state):
    return {n: state[n] for n in ("k_pages", "v_pages", "k_scales", "v_scales", "scores") if state[n] is not None}


def _run_own(state):
    c = state["case"]
    if "ctx" not in state:       # made once, as a serving loop does; the packed arguments belong to the batch and the layer
        from paper_2510_08055_amd import binding
        dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        ctx = binding.KVContext(c["heads"], c["kv_heads"], c["dim"], c["page"], dt, kv_format=c["fmt"], device=DEV)
        state["ctx"] = ctx
        state["batch"] = ctx.pack_batch(state["row_offsets"], state["kv_lens"], state["page_table"])
        if "k_pages" in state:
            state["pages"] = ctx.pack_pages(state["k_pages"], state["v_pages"], state["k_scales"], state["v_scales"])
    ctx, batch = state["ctx"], state["batch"]
    if c["op"] == "masks":
        return list(ctx.moe_tree_masks(state["parents"], batch, words=c["words"], window=c["window"]))
    if c["op"] == "select":
        return list(ctx.moe_kv_select(state["scores"], batch, c["budget"], first=c["first"], recent=c["recent"]))
    if c["op"] in ("accept", "compact"):
        ctx.moe_kv_compact(state["pages"], batch, state["keep"], state["keep_lens"], first=state["first"], scores=state["scores"])
        return _cache(state)
    if c["op"] == "weights":
        return [ctx.moe_kv_weights(state["q"], state["lse"], state["pages"], batch, state["scores"], window=c["window"], decay=c["decay"])]
    ctx.moe_tree_attention(state["q"], state["pages"], batch, state["masks"], positions=state["positions"], window=c["window"],
                           sinks=state["sinks"], out=state["out"], lse=state["lse"])
    return [state["out"], state["lse"]] if c["lse"] else [state["out"]]


def _plain_masks(state):
    """Masks [T, words] (64 bits each) and positions [T]: whom a row reaches by one step, then by two, four, ... steps."""
    c, off, kv = state["case"], state["row_offsets"].long(), state["kv_lens"].long()
    T, W = sum(state["rows"]), c["words"]
    N = min(max(state["rows"]), 64 * W)
    count = off[1:] - off[:-1]
    row = torch.arange(T, device=DEV)
    seq = torch.searchsorted(off[1:], row, right=True)
    i = row - off[seq]
    tree = count <= 64 * W
    # every tree's parents, padded to the largest tree; N stands for none
    at = torch.arange(N, device=DEV)
    real = (at < count[:, None]) & tree[:, None]
    up = torch.where(real, state["parents"].long()[(off[:-1, None] + at).clamp(max=T - 1)], -1)
    up = torch.where((up >= 0) & (up < at), up, N)
    up = torch.cat([up, torch.full_like(up[:, :1], N)], 1)
    reach = torch.eye(N + 1, device=DEV, dtype=torch.bool)[:, :N].expand(len(count), -1, -1).clone()
    reach[:, N] = False
    for _ in range(max(1, (N - 1).bit_length())):
        reach = reach | torch.gather(reach, 1, up[:, :, None].expand(-1, -1, N))
        up = torch.gather(up, 1, up)
    reach = reach[:, :N]
    depth = reach.sum(2) - 1
    if c["window"] > 0:
        reach = reach & (depth[:, :, None] - depth[:, None, :] < c["window"])
    bits = torch.nn.functional.pad(reach, (0, 64 * W - N)).view(len(count), N, W, 64).long()
    words = (bits << torch.arange(64, device=DEV)).sum(3)
    mine = i.clamp(max=N - 1)
    masks = torch.where(tree[seq][:, None], words[seq, mine], 0)
    positions = (kv - count)[seq] + torch.where(tree[seq], depth[seq, mine], i)
    return masks, positions.to(torch.int32)


def _values(codes, scales, page, slot):
    """Cached rows [..., kv_heads, dim] at (page, slot), in fp32."""
    if scales is None:
        return codes[page, :, slot].float()
    x = codes.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).float()
    s = scales[page, :, slot]
    return torch.where(s == BAD_EXP, torch.nan, torch.ldexp(torch.ones_like(s, dtype=torch.float32), s.int() - 127))[..., None] * x


def _plain_scores(state, s0, s1):
    """Scores [n, Hk, R, G, N] of sequences [s0, s1), padded to the most rows and the longest cache among them, minus infinity where a row
    does not see a token; the rows' places, which of them are real, the tokens' pages, slots, and which of them are there."""
    c = state["case"]
    Hq, Hk, D, ps = c["heads"], c["kv_heads"], c["dim"], c["page"]
    R, N, n = max(state["rows"][s0:s1]), max(state["kv"][s0:s1]), s1 - s0
    off, kv = state["row_offsets"].long(), state["kv_lens"][s0:s1].long()
    count = off[s0 + 1:s1 + 1] - off[s0:s1]
    j = torch.arange(N, device=DEV).expand(n, N)
    if c["window"] > 0 and c["op"] == "tree":      # no row sees what lies before the first one's window
        N = min(N, R + c["window"])
        j = (kv - R - c["window"]).clamp(min=0)[:, None] + j[:, :N]
    page = torch.gather(state["page_table"][s0:s1].long(), 1, (j // ps).clamp(max=state["page_table"].shape[1] - 1))
    there = (page >= 0) & (j < kv[:, None])
    page, slot, j = page.clamp(min=0), j % ps, j[:, None, :]
    k = _values(state["k_pages"], state["k_scales"], page, slot).permute(0, 2, 3, 1)            # [n, Hk, D, N]
    i = torch.arange(R, device=DEV)
    real = i < count[:, None]                                                                    # [n, R]
    row = (off[s0:s1, None] + i).clamp(max=state["q"].shape[0] - 1)
    q = state["q"][row].float().view(n, R, Hk, Hq // Hk, D).permute(0, 2, 1, 3, 4).reshape(n, Hk, -1, D)
    p0 = (kv - count)[:, None, None]
    p = p0 + i[:, None]                                                                          # positions of the rows
    seen = j <= p
    if c["op"] == "tree":
        W = c["words"]
        b = (j - p0).clamp(0, 64 * W - 1).expand(n, R, N)
        word = torch.gather(state["masks"][row], 2, b // 64)
        mine = torch.where(j < p0, True, ((word >> (b % 64)) & 1) != 0)
        tree = (count <= 64 * W)[:, None, None]
        seen = torch.where(tree, mine, seen)
        p = torch.where(tree, state["positions"][row].long()[:, :, None], p)
        if c["window"] > 0:
            seen = seen & ((j > p - c["window"]) | (tree & (j >= p0)))
    elif c["window"] > 0:
        seen = seen & (j > p - c["window"])
    seen = seen & there[:, None, :] & real[:, :, None]
    scores = torch.matmul(q, k.contiguous()).mul_(1.0 / math.sqrt(D)).view(n, Hk, R, Hq // Hk, N)
    scores.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    return scores, row, real, page, slot, there


def _plain_attention(state, s0, s1, out, lse):
    c = state["case"]
    Hq, Hk, D, n = c["heads"], c["kv_heads"], c["dim"], s1 - s0
    scores, row, real, page, slot, there = _plain_scores(state, s0, s1)
    R, N = scores.shape[2], scores.shape[4]
    v = torch.where(there[:, :, None, None], _values(state["v_pages"], state["v_scales"], page, slot), 0.0).permute(0, 2, 1, 3)
    m = scores.amax(-1, keepdim=True)
    sink = None
    if state["sinks"] is not None:
        sink = state["sinks"].view(1, Hk, 1, Hq // Hk, 1)
        m = torch.maximum(m, sink)
    m = torch.where(m == -math.inf, 0.0, m)
    w = scores.sub_(m).exp_()
    total = w.sum(-1, keepdim=True)
    if sink is not None:
        total = total + torch.exp(sink - m)
    o = torch.matmul(w.view(n, Hk, -1, N), v.contiguous()).view(n, Hk, R, Hq // Hk, D)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 2, 1, 3, 4).reshape(n, R, Hq, D)
    out[row[real]] = o[real]
    lse[row[real]] = (m + torch.log(total)).squeeze(-1).permute(0, 2, 1, 3).reshape(n, R, Hq)[real]


def _plain_weights(state, s0, s1):
    c = state["case"]
    Hq, Hk, n = c["heads"], c["kv_heads"], s1 - s0
    scores, row, real, page, slot, there = _plain_scores(state, s0, s1)
    R, N = scores.shape[2], scores.shape[4]
    lse = state["lse"][row].view(n, R, Hk, Hq // Hk).permute(0, 2, 1, 3)
    w = scores.sub_(lse[..., None]).exp_().view(n, Hk, -1, N).sum(2).transpose(1, 2)             # [n, N, Hk]
    j = torch.arange(N, device=DEV)
    p0 = (state["kv_lens"].long() - state["row_offsets"].long()[1:] + state["row_offsets"].long()[:-1])[s0:s1]
    old = state["scores"][page, :, slot]
    if c["decay"] == 0.0:
        old = torch.zeros_like(old)
    w = w + torch.where((j < p0[:, None])[:, :, None], c["decay"] * old, 0.0)
    state["scores"][page[there], :, slot[there]] = w[there]


def _plain_select(state):
    """Kept tokens [S, Hk, budget], ascending, -1 behind them, and how many: the first and the recent ones, then by score."""
    c, kv = state["case"], state["kv_lens"].long()
    N, B, ps = max(state["kv"]), c["budget"], c["page"]
    j = torch.arange(N, device=DEV)
    page = state["page_table"].long()[:, j // ps]
    there = (page >= 0) & (j < kv[:, None])
    score = state["scores"][page.clamp(min=0), :, j % ps].permute(0, 2, 1)                       # [S, Hk, N]
    sure = (j < c["first"]) | (j >= kv[:, None] - c["recent"])
    score = torch.where(there[:, None], torch.where(sure[:, None], math.inf, score), -math.inf)
    best = torch.sort(score, dim=2, descending=True, stable=True).indices[:, :, :B]
    lens = kv.clamp(max=B)
    at = torch.arange(best.shape[2], device=DEV)
    best = torch.where(at < lens[:, None, None], best, N).sort(dim=2).values
    keep = torch.where(best < N, best, -1).to(torch.int32)
    return [torch.nn.functional.pad(keep, (0, B - keep.shape[2]), value=-1), lens.to(torch.int32)]


def _plain_compact(state):
    c = state["case"]
    Hk, ps, keep = c["kv_heads"], c["page"], state["keep"].long()
    keep = (keep if c["per_head"] else keep[:, None]).expand(-1, Hk, -1)
    S, M = keep.shape[0], keep.shape[2]
    i = torch.arange(M, device=DEV)
    real = (i < state["keep_lens"][:, None])[:, None].expand(S, Hk, M)
    to = (i + (state["first"].long()[:, None] if state["first"] is not None else 0)).expand(S, M)[:, None].expand(S, Hk, M)[real]
    s = torch.arange(S, device=DEV)[:, None, None].expand(S, Hk, M)[real]
    h = torch.arange(Hk, device=DEV)[None, :, None].expand(S, Hk, M)[real]
    keep = keep[real]
    page, at = state["page_table"].long()[s, keep // ps], state["page_table"].long()[s, to // ps]
    for x in _cache(state).values():
        x = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
        x[at, h, to % ps] = x[page, h, keep % ps]
    return _cache(state)


def exact(case, seed):
    """The definitions in 64 bits, a sequence and a key/value head at a time."""
    c = _full(case)
    if c["op"] in ("masks", "select"):       # whole numbers alone
        return None
    st = prepare(case, seed)
    ps, Hq, Hk, D = c["page"], c["heads"], c["kv_heads"], c["dim"]
    G, fp8, dev = Hq // Hk, c["fmt"] == "fp8", torch.device(DEV)
    table = st["page_table"].cpu().tolist()

    def places(s, tokens):               # of a list of a sequence's tokens
        tokens = torch.as_tensor(tokens)
        return torch.tensor(table[s])[tokens // ps].to(dev), (tokens % ps).to(dev)

    def history(s, h, n, what):          # the first n tokens of a sequence
        page, slot = places(s, torch.arange(n))
        x = st[what + "_pages"][:, h]
        x = (x.view(torch.uint8)[page, slot].view(torch.float8_e4m3fn).float() if fp8 else x[page, slot]).double()
        return x * torch.pow(2.0, st[what + "_scales"][:, h][page, slot].double() - 127.0)[:, None] if fp8 else x

    if c["op"] in ("accept", "compact"):
        new = {}
        keep, lens = st["keep"].cpu(), st["keep_lens"].cpu().tolist()
        start = st["first"].cpu().tolist() if st["first"] is not None else [0] * len(lens)
        for name, x in _cache(st).items():
            if x.dtype == torch.uint8:
                new[name] = None
                continue
            y = x.float().double()
            was = y.clone()
            for s, n in enumerate(lens):
                page, slot = places(s, torch.arange(start[s], start[s] + n))
                for h in range(Hk):
                    a, b = places(s, (keep[s, h] if c["per_head"] else keep[s])[:n].long())
                    y[page, h, slot] = was[a, h, b]
            new[name] = y
        return new
    T = sum(st["rows"])
    parents = st["parents"].cpu().tolist() if c["op"] == "tree" else []
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device=dev)
    lse = torch.zeros(T, Hq, dtype=torch.float64, device=dev)
    scores = st["scores"].double() if c["op"] == "weights" else None
    t = 0
    for s, (n, kv) in enumerate(zip(st["rows"], st["kv"])):
        at, j = torch.arange(kv - n, kv, device=dev)[:, None], torch.arange(kv, device=dev)[None]
        hidden = j > at
        if c["window"]:
            hidden = hidden | (at - j >= c["window"])
        if _is_tree(c, n):               # path by path
            paths = []
            for i in range(n):
                up = parents[t + i]
                paths.append((paths[up] if up >= 0 else []) + [i])
            sees = torch.zeros(n, kv, dtype=torch.bool)
            for i, path in enumerate(paths):
                reach = c["window"] or kv + n
                sees[i, max(0, kv - n + len(path) - reach):kv - n] = True
                sees[i, [kv - n + a for a in path[-reach:]]] = True
            hidden = ~sees.to(dev)
        for h in range(Hk):
            k = history(s, h, kv, "k")
            v = history(s, h, kv, "v") if c["op"] == "tree" else None
            total = torch.zeros(kv, dtype=torch.float64, device=dev)
            for g in range(h * G, (h + 1) * G):
                z = (st["q"][t:t + n, g].double() @ k.T) / math.sqrt(D)
                z[hidden] = -math.inf
                if c["op"] == "weights":
                    total += torch.exp(z - st["lse"][t:t + n, g].double()[:, None]).sum(0)
                    continue
                if c["sinks"]:
                    z = torch.cat([z, st["sinks"][g].double().expand(n, 1)], 1)
                lse[t:t + n, g] = torch.logsumexp(z, 1)
                out[t:t + n, g] = torch.softmax(z, 1)[:, :kv] @ v
            if c["op"] == "weights":
                page, slot = places(s, torch.arange(kv))
                old = scores[page, h, slot] * c["decay"]
                old[kv - n:] = 0.0
                scores[page, h, slot] = old + total
        t += n
    if c["op"] == "weights":
        return [scores]
    return [out, lse] if c["lse"] else [out]
