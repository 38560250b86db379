"""The paged key/value cache and its attention in 64 bits, a sequence and a head at a time, and how far off results may be."""
import math

import torch

EPS = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step of a rounding, relative


def quantised(x):
    """Codes and scale bytes of rows x [..., dim]: the smallest 2^e, e >= -100, with amax <= 448 * 2^e (2^-9 for zeros)."""
    x = x.double().cpu()
    amax = x.abs().amax(-1)
    codes, scales = torch.empty(x.shape, dtype=torch.uint8), torch.empty(amax.shape, dtype=torch.uint8)
    for i in range(amax.numel()):
        a, row = float(amax.view(-1)[i]), x.reshape(-1, x.shape[-1])[i]
        if not math.isfinite(a):
            codes.view(-1, x.shape[-1])[i], scales.view(-1)[i] = 0x7f, 255
            continue
        e = -9
        if a > 0:
            e = -100
            while a > 448.0 * 2.0 ** e:
                e += 1
        codes.view(-1, x.shape[-1])[i] = (row * 2.0 ** -e).float().to(torch.float8_e4m3fn).view(torch.uint8)
        scales.view(-1)[i] = e + 127
    return codes, scales


def worth(codes, scales):
    """What codes and scale bytes stand for, in 64 bits."""
    v = codes.view(torch.float8_e4m3fn).float().double()
    s = torch.where(scales == 255, math.nan, torch.pow(2.0, scales.double() - 127.0))
    return v * s.unsqueeze(-1)


def history(pages, scales, table, n_tokens, h, page):
    """The first n_tokens of a sequence (table: its row of the page table) for one head, and which of them are there."""
    n_pages = pages.shape[0]
    pos = torch.arange(n_tokens, device=pages.device)
    ids = torch.full((n_tokens,), -1, dtype=torch.long, device=pages.device)
    inside = pos // page < table.numel()
    ids[inside] = table.long()[pos[inside] // page]
    here = (ids >= 0) & (ids < n_pages)
    i, slot = ids.clamp(0, n_pages - 1), pos % page
    x = worth(pages.view(torch.uint8)[i, h, slot], scales[i, h, slot]) if scales is not None else pages[i, h, slot].double()
    x[~here] = 0
    return x, here


def attention(q, pages, offsets, lens, table, page, causal=True, window=0, sinks=None):
    """out, lse and the bounds of their errors for q [T, heads, dim] (the kernels' rounding points counted)."""
    k_pages, v_pages, k_scales, v_scales = pages
    T, heads, dim = q.shape
    hk = k_pages.shape[1]
    out = torch.zeros(T, heads, dim, dtype=torch.float64, device=q.device)
    lse = torch.full((T, heads), -math.inf, dtype=torch.float64, device=q.device)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    u = 2.0 ** -24
    for s in range(len(lens)):
        r0, r1, kv = offsets[s], offsets[s + 1], min(lens[s], table.shape[1] * page)
        if r1 == r0:
            continue
        pos = torch.arange(kv - (r1 - r0), kv, device=q.device)[:, None]
        j = torch.arange(kv, device=q.device)[None]
        for h in range(hk):
            k, here = history(k_pages, k_scales, table[s], kv, h, page)
            v, _ = history(v_pages, v_scales, table[s], kv, h, page)
            seen = here[None] & torch.ones_like(pos, dtype=torch.bool)
            if causal:
                seen = seen & (j <= pos)
            if window > 0:
                seen = seen & (j > pos - window)
            some = seen.any(0)
            k = torch.where(some[:, None], k, 0.0)
            strange = ~torch.isfinite(v)
            vf = torch.where(strange, 0.0, v)
            g = heads // hk
            for head in range(h * g, (h + 1) * g):
                qh = q[r0:r1, head].double()
                z = torch.where(seen, (qh @ k.T) / math.sqrt(dim), -math.inf)
                size = torch.where(seen, (qh.abs() @ k.abs().T) / math.sqrt(dim), 0.0).nan_to_num(0.0, 0.0, 0.0)
                dz = (dim + 8) * u * size.amax(1) if kv else torch.zeros(r1 - r0, dtype=torch.float64, device=q.device)
                top = z.amax(1) if kv else torch.full((r1 - r0,), -math.inf, dtype=torch.float64, device=q.device)
                if sinks is not None:
                    top = torch.maximum(top, sinks[head].double())
                top = torch.where(top == -math.inf, 0.0, top)
                w = torch.exp(z - top[:, None])
                total = w.sum(1) + (torch.exp(sinks[head].double() - top) if sinks is not None else 0.0)
                w = torch.where(total[:, None] > 0, w / total[:, None], torch.where(total[:, None] == 0, 0.0, total[:, None]))
                o = w @ vf
                o = torch.where((seen.double() @ strange.double()) > 0, math.nan, o)
                size = w @ vf.abs()
                out[r0:r1, head] = o
                lse[r0:r1, head] = torch.where(total > 0, top + torch.log(total), torch.where(total == 0, -math.inf, total))
                # exponentials are off by twice the scores' error, the reference's rounding and their own; sums by a step a term
                rel = 2 * dz + 2 * top.abs() * 4 * u + (kv + 64) * u
                stored = EPS[torch.bfloat16] if q.dtype == torch.bfloat16 else 0.0
                tol[r0:r1, head] = EPS[q.dtype] * o.abs() * (1 + 2.0 ** -7) + (rel + stored)[:, None] * size + 1e-30 \
                    if torch.is_tensor(rel) else 0
                ltol[r0:r1, head] = rel + 8 * u * (1 + top.abs())
    return out, lse, tol, ltol


def assert_within(got, ref, tol, what=""):
    got, ref = got.double(), ref.to(got.device)
    nan = torch.isnan(ref)
    assert not torch.isfinite(got[nan]).any(), f"{what}: finite where the result has no finite value"
    same = (got == ref) | nan
    err = torch.where(same, 0.0, (got - ref).abs())
    bad = ~(err <= tol.to(got.device))
    if bad.any():
        at = bad.nonzero()[0].tolist()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {at}: {got[tuple(at)].item()!r} for "
                             f"{ref[tuple(at)].item()!r}, bound {tol[tuple(at)].item():.3e}")


class Batch:
    """A cache with random pages in random order, its descriptors, and the new tokens' rows as views of one fused tensor.

    Whatever no token needs (pages, slots past a sequence's end, scale bytes there) is NaN."""

    def __init__(self, rows, kv, heads, kv_heads, dim, page, dtype=torch.bfloat16, fmt="", seed=0, device="cuda:0", dropped=(),
                 extra_pages=3):
        g = torch.Generator().manual_seed(seed)
        self.rows, self.kv, self.page, self.dtype, self.fmt, self.device = rows, kv, page, dtype, fmt, device
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.offsets = [0]
        for n in rows:
            self.offsets.append(self.offsets[-1] + n)
        T = self.offsets[-1]
        need = [-(-k // page) for k in kv]
        n_pages = sum(need) + extra_pages
        order = torch.randperm(n_pages, generator=g).tolist()
        self.table = torch.full((len(kv), max(need + [0]) + 1), -1, dtype=torch.int32)
        used = torch.zeros(n_pages, page, dtype=torch.bool)
        for s, n in enumerate(need):
            for i in range(n):
                at = order.pop()
                used[at, :min(page, kv[s] - i * page)] = True
                if (s, i) not in dropped:
                    self.table[s, i] = at
        used = used[:, None, :, None].expand(n_pages, kv_heads, page, 1)
        loud = torch.exp(0.5 * torch.randn(kv_heads, 1, dim, generator=g))

        def pages(channel):
            x = torch.randn(n_pages, kv_heads, page, dim, generator=g) * channel
            if fmt == "fp8":
                a = x.abs().amax(-1, keepdim=True)
                e = torch.ceil(torch.log2(a / 448.0)).clamp(min=-100)
                codes = torch.where(used, (x * torch.pow(2.0, -e)).clamp(-448, 448), math.nan).to(torch.float8_e4m3fn)
                return codes.to(device), torch.where(used, e + 127, 255.0).squeeze(-1).to(torch.uint8).to(device)
            return torch.where(used, x, math.nan).to(dtype).to(device), None

        self.k_pages, self.k_scales = pages(loud)
        self.v_pages, self.v_scales = pages(1.0)
        fused = torch.randn(T, (heads + 2 * kv_heads) * dim, generator=g).to(dtype).to(device)
        self.q = fused[:, :heads * dim].unflatten(1, (heads, dim))
        self.k = fused[:, heads * dim:(heads + kv_heads) * dim].unflatten(1, (kv_heads, dim))
        self.v = fused[:, (heads + kv_heads) * dim:].unflatten(1, (kv_heads, dim))
        self.table = self.table.to(device)
        self.row_offsets = torch.tensor(self.offsets, dtype=torch.int32, device=device)
        self.kv_lens = torch.tensor(kv, dtype=torch.int32, device=device)
        self.T = T

    def pages(self):
        return self.k_pages, self.v_pages, self.k_scales, self.v_scales

    def context(self, lib):
        ctx = lib.KVContext(self.heads, self.kv_heads, self.dim, self.page, self.dtype, kv_format=self.fmt, device=self.device)
        return ctx, ctx.pack_pages(*self.pages()), ctx.pack_batch(self.row_offsets, self.kv_lens, self.table)

    def reference(self, causal=True, window=0, sinks=None):
        return attention(self.q, self.pages(), self.offsets, self.kv, self.table, self.page, causal, window, sinks)
