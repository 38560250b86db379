"""The paged key/value cache and the attention that reads it, as a list of cases to measure.

Three operators of a hybrid batch (decode rows beside prompt rows): `moe_kv_append` writes the new tokens' keys and
values into the pages of a cache, as they are or as FP8 codes with a scale per token and head; `moe_kv_gather` reads
rows back; `moe_paged_attention` attends from the new tokens to everything their sequences hold.  A case is one call.
`run` is either the framework's call (`own`) or the same in elementary torch operations in fp32.

The batch sizes are those of the repository's workloads: 1 to 256 decode rows, chunks of 512 tokens, prompts of up to
8192; the heads are generic (groups of 1 to 16 query heads to a key/value head, 64 to 128 wide, 256 in a few draws).
"""
import math

import torch

own = False

DEV = "cuda:0"

# What a case may leave out.  D sequences of `rows` new tokens each, with kv_lo to kv_hi tokens in the cache (spread over
# the logarithm), then `prompts` sequences of P / 2 to P new tokens (P for a single one) behind `past` cached tokens.
# fmt: "" (the cache holds dtype) or "fp8".  dropped: pages that lie wholly before every row's window are given back.
DEFAULTS = {"heads": 32, "kv_heads": 4, "dim": 128, "page": 16, "dtype": "bf16", "fmt": "", "D": 0, "rows": 1,
            "kv_lo": 1, "kv_hi": 1, "prompts": 0, "P": 0, "past": 0, "window": 0, "dropped": False, "sinks": False,
            "causal": True, "lse": False}

WIDE = {"heads": 32, "kv_heads": 4, "dim": 128}      # eight query heads to a key/value head
HALF = {"heads": 64, "kv_heads": 8, "dim": 64}       # the same groups, half as wide
QUAD = {"heads": 32, "kv_heads": 8, "dim": 128}      # groups of four
FP8_MAX, MIN_EXP, BAD_EXP = 448.0, -100, 255


def listed():
    return [
        # a decode step writes one token of 32 sequences: nothing but latency
        {"name": "append_step", "op": "append", **WIDE, "D": 32, "kv_lo": 64, "kv_hi": 1024},
        # layered prefill writes a whole 8192-token prompt and 128 decode rows, quantised
        {"name": "append_prompt_fp8", "op": "append", **WIDE, "page": 64, "fmt": "fp8", "D": 128, "kv_lo": 16, "kv_hi": 256,
         "prompts": 1, "P": 8192},
        # a few finished sequences are read back whole for a prefix store, odd lengths
        {"name": "gather_odd", "op": "gather", **QUAD, "D": 3, "kv_lo": 301, "kv_hi": 1999},
        # 16 quantised histories are read back whole
        {"name": "gather_fp8", "op": "gather", **HALF, "page": 32, "fmt": "fp8", "D": 16, "kv_lo": 1024, "kv_hi": 8192},
        # one user's decode step early in a reply: launches and latency
        {"name": "decode_one", "op": "attention", **WIDE, "D": 1, "kv_lo": 700, "kv_hi": 700},
        # the largest usual decode batch, ragged histories of 512 to 8192 tokens: streams the cache
        {"name": "decode_batch", "op": "attention", **WIDE, "D": 128, "kv_lo": 512, "kv_hi": 8192},
        # long histories in a quantised cache, four drafted tokens to a sequence
        {"name": "decode_draft_fp8", "op": "attention", **QUAD, "page": 64, "fmt": "fp8", "D": 24, "rows": 4, "kv_lo": 2048,
         "kv_hi": 32768},
        # a layer with a sliding window and sinks, whose cache has given old pages back: 256 decode rows
        {"name": "decode_window", "op": "attention", **HALF, "D": 256, "kv_lo": 100, "kv_hi": 4096, "window": 128,
         "dropped": True, "sinks": True},
        # chunked prefill: the sixteenth chunk of 512 tokens re-reads 7680 cached ones, beside 32 decode rows
        {"name": "chunk", "op": "attention", **WIDE, "D": 32, "kv_lo": 512, "kv_hi": 4096, "prompts": 1, "P": 512, "past": 7680},
        # layered prefill: the whole 8192-token prompt at once, beside 128 decode rows
        {"name": "prompt", "op": "attention", **WIDE, "D": 128, "kv_lo": 64, "kv_hi": 1024, "prompts": 1, "P": 8192},
        # ragged prompts side by side over a quantised cache, narrow heads
        {"name": "prompts_fp8", "op": "attention", **HALF, "page": 32, "fmt": "fp8", "prompts": 5, "P": 1900, "past": 77},
        # the fp32 path: a small model's prompt, with the log-sum-exp that joins it to another part
        {"name": "prompt_f32", "op": "attention", "heads": 8, "kv_heads": 2, "dim": 32, "dtype": "f32", "prompts": 2, "P": 192,
         "past": 13, "lse": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges above; it costs no more than the largest listed one."""
    kind = rng.choice(["append", "append", "gather", "decode", "decode", "decode", "draft", "window", "chunk", "prompt",
                       "prompts", "f32", "full"])
    kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8, 16])
    dim = rng.choice([64, 64, 80, 96, 112, 128, 128, 128, 256])
    c = {"heads": kv_heads * group, "kv_heads": kv_heads, "dim": dim, "page": rng.choice([8, 16, 16, 32, 64, 128]),
         "fmt": rng.choice(["", "fp8"])}
    if kind == "append":
        c.update(op="append", D=_log_int(rng, 1, 256), kv_lo=1, kv_hi=500, prompts=rng.choice([0, 1, 2]),
                 P=_log_int(rng, 2, 4096), past=rng.randint(0, 300), dtype=rng.choice(["bf16", "bf16", "f32"]))
    elif kind == "gather":
        c.update(op="gather", D=_log_int(rng, 1, 24), kv_lo=_log_int(rng, 1, 200), kv_hi=_log_int(rng, 201, 4000),
                 dtype=rng.choice(["bf16", "bf16", "f32"]))
    elif kind == "decode":
        hi = _log_int(rng, 16, 8192)
        c.update(op="attention", D=_log_int(rng, 1, 128), kv_lo=rng.randint(1, 16), kv_hi=hi)
    elif kind == "draft":
        c.update(op="attention", D=_log_int(rng, 1, 32), rows=rng.randint(2, 9), kv_lo=rng.randint(9, 64),
                 kv_hi=_log_int(rng, 64, 8192))
    elif kind == "window":
        c.update(op="attention", D=_log_int(rng, 1, 256), kv_lo=rng.randint(1, 64), kv_hi=_log_int(rng, 64, 4096),
                 window=_log_int(rng, 8, 1024), dropped=rng.random() < 0.5, sinks=rng.random() < 0.7,
                 prompts=rng.choice([0, 0, 1]), P=rng.randint(2, 1500))
    elif kind == "chunk":
        c.update(op="attention", D=rng.randint(0, 32), kv_lo=16, kv_hi=_log_int(rng, 16, 2048), prompts=rng.choice([1, 1, 2]),
                 P=rng.choice([256, 512, 512, 1024, rng.randint(33, 1100)]), past=_log_int(rng, 1, 6000), sinks=rng.random() < 0.2)
    elif kind == "prompt":
        c.update(op="attention", D=rng.randint(0, 64), kv_lo=16, kv_hi=_log_int(rng, 16, 1024), prompts=1, P=_log_int(rng, 17, 4000),
                 lse=rng.random() < 0.2)
    elif kind == "prompts":
        c.update(op="attention", prompts=rng.randint(2, 6), P=_log_int(rng, 16, 1500), past=rng.randint(0, 200))
    elif kind == "full":
        c.update(op="attention", D=rng.randint(0, 8), kv_lo=8, kv_hi=500, prompts=rng.randint(1, 3), P=_log_int(rng, 8, 1000),
                 causal=False)
    else:
        c.update(op="attention", dtype="f32", D=rng.randint(0, 16), kv_lo=1, kv_hi=600, prompts=rng.choice([0, 1, 2]),
                 P=_log_int(rng, 4, 500), past=rng.randint(0, 50), lse=rng.random() < 0.5)
        if c["D"] + c["prompts"] == 0:
            c["D"] = 1
    return c


def _full(case):
    return {**DEFAULTS, **case}


def _spread(i):
    return (i + 1) * 0.6180339887498949 % 1.0


def _lens(c):
    """(new rows, tokens in the cache with them) of every sequence."""
    rows, kv = [], []
    for i in range(c["D"]):
        n = int(round(c["kv_lo"] * (c["kv_hi"] / c["kv_lo"]) ** _spread(i)))
        rows.append(n if c["op"] == "gather" else c["rows"])
        kv.append(max(n, rows[-1]))
    for i in range(c["prompts"]):
        n = c["P"] if c["prompts"] == 1 else max(1, int(c["P"] * (0.5 + 0.5 * _spread(i))))
        rows.append(n)
        kv.append(c["past"] + n)
    return rows, kv


def _first_kept(c, n, kv):
    """First position of a sequence that some row sees."""
    return max(0, kv - n + 1 - c["window"]) if c["window"] > 0 else 0


def work(case):
    c = _full(case)
    rows, kv = _lens(c)
    esz = 4 if c["dtype"] == "f32" else 2
    token = 2.0 * c["kv_heads"] * ((c["dim"] + 1) if c["fmt"] == "fp8" else c["dim"] * esz)      # K and V of a cached token
    if c["op"] != "attention":
        return {"bytes": sum(rows) * (token + 2.0 * c["kv_heads"] * c["dim"] * esz), "flops": 0}
    nbytes = 2.0 * sum(rows) * c["heads"] * c["dim"] * esz + (sum(rows) * c["heads"] * 4.0 if c["lse"] else 0.0)
    pairs = 0
    for n, k in zip(rows, kv):
        nbytes += (k - _first_kept(c, n, k)) * token
        if not c["causal"]:
            pairs += n * k
        else:
            w = c["window"] or k
            past = k - n
            full = max(0, min(n, w - past))         # rows whose window reaches back to position 0
            pairs += full * past + full * (full + 1) // 2 + (n - full) * w
    return {"bytes": nbytes, "flops": 4.0 * c["heads"] * c["dim"] * pairs}


def _quantised(x):
    """FP8 codes and scale bytes of rows x [..., dim] (fp32): the scale 2^e is the smallest power of two, e >= -100, that
    keeps the row within the codes' range; a row with a value that is not finite is NaN throughout."""
    amax = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=MIN_EXP)
    bad = ~torch.isfinite(amax)
    codes = torch.where(bad, torch.nan, torch.ldexp(x, -e)).to(torch.float8_e4m3fn)
    return codes, torch.where(bad, BAD_EXP, e + 127).squeeze(-1).to(torch.uint8)


def prepare(case, seed):
    """A cache with its page table, the batch's lengths, and the new tokens' projections as one fused tensor's views."""
    c = _full(case)
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    rows, kv = _lens(c)
    S, T, ps, Hq, Hk, D = len(rows), sum(rows), c["page"], c["heads"], c["kv_heads"], c["dim"]
    need = [-(-k // ps) for k in kv]
    max_pages = max(need) + 1
    n_pages = sum(need) + 7

    # pages are handed out in random order; entries that no token needs are -1
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    counts = torch.tensor(need, device=DEV)
    first = torch.cumsum(counts, 0) - counts
    at = torch.arange(max_pages, device=DEV)
    gone = torch.tensor([_first_kept(c, n, k) // ps if c["dropped"] else 0 for n, k in zip(rows, kv)], device=DEV)
    held = (at < counts[:, None]) & (at >= gone[:, None])
    table = torch.where(held, order[(first[:, None] + at).clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous()

    loud = torch.exp(0.5 * torch.randn(Hk, 1, D, generator=g, device=DEV))       # some channels of the keys are louder than others

    def pages(channel):
        x = torch.randn(n_pages, Hk, ps, D, generator=g, device=DEV) * channel
        return _quantised(x.to(dt).float()) if c["fmt"] == "fp8" else (x.to(dt), None)

    k_pages, k_scales = pages(loud)
    v_pages, v_scales = pages(1.0)
    qkv = torch.randn(T, (Hq + 2 * Hk) * D, generator=g, device=DEV)
    qkv[:, Hq * D:(Hq + Hk) * D].view(T, Hk, D).mul_(loud.squeeze(1))
    qkv = qkv.to(dt)
    offsets = [0]
    for n in rows:
        offsets.append(offsets[-1] + n)
    st = {"case": c, "k_pages": k_pages, "v_pages": v_pages, "k_scales": k_scales, "v_scales": v_scales, "page_table": table,
          "row_offsets": torch.tensor(offsets, dtype=torch.int32, device=DEV),
          "kv_lens": torch.tensor(kv, dtype=torch.int32, device=DEV), "rows": rows, "kv": kv,
          "q": qkv[:, :Hq * D].unflatten(1, (Hq, D)), "k": qkv[:, Hq * D:(Hq + Hk) * D].unflatten(1, (Hk, D)),
          "v": qkv[:, (Hq + Hk) * D:].unflatten(1, (Hk, D)),
          "sinks": torch.randn(Hq, generator=g, device=DEV) if c["sinks"] else None}
    if c["op"] == "attention":
        st["out"] = torch.empty(T, Hq, D, dtype=dt, device=DEV)
        st["lse"] = torch.empty(T, Hq, device=DEV) if c["lse"] else None
    elif c["op"] == "gather":
        st["k_out"], st["v_out"] = (torch.empty(T, Hk, D, dtype=dt, device=DEV) for _ in range(2))
    return st


def run(state):
    c = state["case"]
    if own:
        return _run_own(state)
    if c["op"] == "append":
        return _plain_append(state)
    if c["op"] == "gather":
        return _plain_gather(state)
    T = sum(state["rows"])
    out = torch.empty(T, c["heads"], c["dim"], device=DEV)
    lse = torch.empty(T, c["heads"], device=DEV)
    # the decode rows and the prompts have lengths of their own: each padded to its longest
    if c["D"]:
        _plain_attention(state, 0, c["D"], out, lse)
    if c["prompts"]:
        _plain_attention(state, c["D"], c["D"] + c["prompts"], out, lse)
    out = out.to(state["q"].dtype)
    return [out, lse] if c["lse"] else [out]


def _cache(state):
    return {n: state[n] for n in ("k_pages", "v_pages", "k_scales", "v_scales") if state[n] is not None}


def _run_own(state):
    c = state["case"]
    if "ctx" not in state:       # made once, as a serving loop does; the packed arguments belong to the batch and the layer
        from paper_2510_08055_amd import binding
        dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        ctx = binding.KVContext(c["heads"], c["kv_heads"], c["dim"], c["page"], dt, kv_format=c["fmt"], device=DEV)
        state["ctx"] = ctx
        state["pages"] = ctx.pack_pages(state["k_pages"], state["v_pages"], state["k_scales"], state["v_scales"])
        state["batch"] = ctx.pack_batch(state["row_offsets"], state["kv_lens"], state["page_table"])
    ctx, pages, batch = state["ctx"], state["pages"], state["batch"]
    if c["op"] == "append":
        ctx.moe_kv_append(state["k"], state["v"], pages, batch)
        return _cache(state)
    if c["op"] == "gather":
        return list(ctx.moe_kv_gather(pages, batch, k=state["k_out"], v=state["v_out"]))
    ctx.moe_paged_attention(state["q"], pages, batch, causal=c["causal"], window=c["window"], sinks=state["sinks"],
                            out=state["out"], lse=state["lse"])
    return [state["out"], state["lse"]] if c["lse"] else [state["out"]]


def _row_places(state):
    """(page, slot) of every row of the batch: the new tokens are the last ones of their sequences."""
    off, T = state["row_offsets"].long(), sum(state["rows"])
    row = torch.arange(T, device=DEV)
    seq = torch.searchsorted(off[1:], row, right=True)
    pos = state["kv_lens"][seq].long() - off[seq + 1] + row
    ps = state["case"]["page"]
    return state["page_table"][seq, pos // ps].long(), pos % ps


def _plain_append(state):
    page, slot = _row_places(state)
    k, v = state["k"].float(), state["v"].float()
    if state["case"]["fmt"] != "fp8":
        state["k_pages"][page, :, slot] = k.to(state["k_pages"].dtype)
        state["v_pages"][page, :, slot] = v.to(state["v_pages"].dtype)
        return _cache(state)
    kc, ks = _quantised(k)
    vc, vs = _quantised(v)
    state["k_pages"].view(torch.uint8)[page, :, slot] = kc.view(torch.uint8)
    state["v_pages"].view(torch.uint8)[page, :, slot] = vc.view(torch.uint8)
    state["k_scales"][page, :, slot] = ks
    state["v_scales"][page, :, slot] = vs
    return _cache(state)


def _values(codes, scales, page, slot):
    """Cached rows [..., kv_heads, dim] at (page, slot), in fp32."""
    if scales is None:
        return codes[page, :, slot].float()
    x = codes.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).float()
    s = scales[page, :, slot]
    return torch.where(s == BAD_EXP, torch.nan, torch.ldexp(torch.ones_like(s, dtype=torch.float32), s.int() - 127))[..., None] * x


def _plain_gather(state):
    page, slot = _row_places(state)
    dt = state["k_out"].dtype
    return [_values(state["k_pages"], state["k_scales"], page, slot).to(dt),
            _values(state["v_pages"], state["v_scales"], page, slot).to(dt)]


def _plain_attention(state, s0, s1, out, lse):
    """Attention of sequences [s0, s1), padded to the most rows and the longest cache among them."""
    c = state["case"]
    Hq, Hk, D, ps = c["heads"], c["kv_heads"], c["dim"], c["page"]
    R, N, n = max(state["rows"][s0:s1]), max(state["kv"][s0:s1]), s1 - s0
    off, kv = state["row_offsets"].long(), state["kv_lens"][s0:s1].long()
    count = off[s0 + 1:s1 + 1] - off[s0:s1]
    j = torch.arange(N, device=DEV).expand(n, N)
    if c["window"] > 0:      # no row sees what lies before the first one's window
        N = min(N, R + c["window"])
        j = (kv - R - c["window"]).clamp(min=0)[:, None] + j[:, :N]
    page = torch.gather(state["page_table"][s0:s1].long(), 1, (j // ps).clamp(max=state["page_table"].shape[1] - 1))
    there = (page >= 0) & (j < kv[:, None])
    page, slot, j = page.clamp(min=0), j % ps, j[:, None, :]
    k = _values(state["k_pages"], state["k_scales"], page, slot).permute(0, 2, 3, 1)            # [n, Hk, D, N]
    v = torch.where(there[:, :, None, None], _values(state["v_pages"], state["v_scales"], page, slot), 0.0).permute(0, 2, 1, 3)
    i = torch.arange(R, device=DEV)
    real = i < count[:, None]                                                                   # [n, R]
    row = (off[s0:s1, None] + i).clamp(max=out.shape[0] - 1)
    q = state["q"][row].float().view(n, R, Hk, Hq // Hk, D).permute(0, 2, 1, 3, 4).reshape(n, Hk, -1, D)
    p = kv[:, None] - count[:, None] + i                                                        # positions of the rows
    seen = there[:, None, :]
    if c["causal"]:
        seen = seen & (j <= p[:, :, None])
    if c["window"] > 0:
        seen = seen & (j > p[:, :, None] - c["window"])
    scores = torch.matmul(q, k.contiguous()).mul_(1.0 / math.sqrt(D)).view(n, Hk, R, Hq // Hk, N)
    scores.masked_fill_(~seen[:, None, :, None, :], -math.inf)
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


def exact(case, seed):
    """The definition in 64 bits, a sequence and a key/value head at a time."""
    c, st = _full(case), prepare(case, seed)
    ps, Hq, Hk, D = c["page"], c["heads"], c["kv_heads"], c["dim"]
    G, fp8 = Hq // Hk, c["fmt"] == "fp8"
    table = st["page_table"].cpu().tolist()

    def worth(x, s):                     # cached values and the bytes of their scales, as numbers
        x = x.to(torch.float64)
        return x if s is None else x * torch.pow(2.0, s.to(torch.float64) - 127.0).unsqueeze(-1)

    def history(s, h, n, what):          # the first n tokens of a sequence and which of them are there
        ids = torch.tensor(table[s][:-(-n // ps)], device=DEV)
        here = ids >= 0
        x = st[what + "_pages"][:, h].view(torch.uint8)[ids.clamp(min=0)].view(torch.float8_e4m3fn).float() if fp8 else \
            st[what + "_pages"][:, h][ids.clamp(min=0)]
        x = worth(x, st[what + "_scales"][:, h][ids.clamp(min=0)] if fp8 else None)
        x = torch.where(here[:, None, None], x, 0.0)
        return x.reshape(-1, D)[:n], here.repeat_interleave(ps)[:n]

    if c["op"] == "append":
        new = {}
        for what in ("k", "v"):
            x = st[what].to(torch.float64)
            pages = st[what + "_pages"]
            pages = pages.float().double() if fp8 else pages.double()
            if fp8:                      # what a code stands for before it is rounded: the value over its row's scale
                top = x.abs().amax(-1, keepdim=True)
                e = torch.ceil(torch.log2(top / FP8_MAX))
                e = torch.where(top <= FP8_MAX * torch.pow(2.0, e - 1), e - 1, torch.where(top > FP8_MAX * torch.pow(2.0, e), e + 1, e))
                x = x / torch.pow(2.0, e.clamp(min=MIN_EXP))
            t = 0
            for s, (n, kv) in enumerate(zip(st["rows"], st["kv"])):
                pos = torch.arange(kv - n, kv)
                ids = torch.tensor(table[s])[pos // ps]
                pages[ids.to(DEV), :, (pos % ps).to(DEV)] = x[t:t + n]
                t += n
            new[what + "_pages"] = pages
            if fp8:
                new[what + "_scales"] = None
        return new
    if c["op"] == "gather":
        got = []
        for what in ("k", "v"):
            got.append(torch.cat([torch.stack([history(s, h, kv, what)[0][kv - n:] for h in range(Hk)], 1)
                                  for s, (n, kv) in enumerate(zip(st["rows"], st["kv"]))]))
        return got
    out = torch.zeros(sum(st["rows"]), Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(sum(st["rows"]), Hq, dtype=torch.float64, device=DEV)
    t = 0
    for s, (n, kv) in enumerate(zip(st["rows"], st["kv"])):
        at, j = torch.arange(kv - n, kv, device=DEV)[:, None], torch.arange(kv, device=DEV)[None]
        for h in range(Hk):
            k, here = history(s, h, kv, "k")
            v, _ = history(s, h, kv, "v")
            hidden = ~here[None] | ((j > at) if c["causal"] else torch.zeros_like(j > at))
            if c["window"]:
                hidden = hidden | (at - j >= c["window"])
            for g in range(h * G, (h + 1) * G):
                z = (st["q"][t:t + n, g].double() @ k.T) / math.sqrt(D)
                z[hidden] = -math.inf
                if c["sinks"]:
                    z = torch.cat([z, st["sinks"][g].double().expand(n, 1)], 1)
                lse[t:t + n, g] = torch.logsumexp(z, 1)
                out[t:t + n, g] = torch.softmax(z, 1)[:, :kv].nan_to_num(0.0) @ v
        t += n
    return [out, lse] if c["lse"] else [out]
