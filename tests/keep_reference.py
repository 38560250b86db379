"""Trees of drafted tokens, accumulated attention weights, and what a cache keeps, by their definitions in 64 bits or in plain Python."""
import math

import torch

from kv_reference import EPS, history

U = 2.0 ** -24


def paths(parents):
    """The path of every row of a tree, from its root; a parent that does not come before its child is none."""
    got = []
    for i, up in enumerate(parents):
        got.append((got[up] if 0 <= up < i else []) + [i])
    return got


def tree_masks(parents, offsets, lens, words, window):
    """Masks [T, words] as signed 64-bit integers, and positions [T]."""
    T = len(parents)
    masks, positions = torch.zeros(T, words, dtype=torch.int64), torch.zeros(T, dtype=torch.int32)
    for s, kv in enumerate(lens):
        r0, n = offsets[s], offsets[s + 1] - offsets[s]
        p0 = max(kv, 0) - n
        if n > 64 * words:
            positions[r0:r0 + n] = torch.arange(p0, p0 + n)
            continue
        for i, path in enumerate(paths(parents[r0:r0 + n])):
            positions[r0 + i] = p0 + len(path) - 1
            for j in path[-window:] if window else path:
                bit = 1 << (j % 64)
                masks[r0 + i, j // 64] |= bit - (1 << 64) if bit >= 1 << 63 else bit
    return masks, positions


def seen_by_masks(masks, positions, n, kv, words, window):
    """Which of the tokens before kv the rows [n] of a sequence see, by their masks (a list of lists of words) and positions."""
    p0 = kv - n
    sees = torch.zeros(n, max(kv, 0), dtype=torch.bool)
    for i in range(n):
        if n > 64 * words:
            lo, hi = (max(0, p0 + i - window + 1) if window else 0), p0 + i + 1
            if hi > lo:
                sees[i, lo:hi] = True
            continue
        pos = min(max(positions[i], p0), kv - 1) if window else 0
        lo = max(0, pos - window + 1) if window else 0
        if p0 > lo:
            sees[i, lo:p0] = True
        for j in range(n):
            if (masks[i][j // 64] >> (j % 64)) & 1 and p0 + j >= 0:
                sees[i, p0 + j] = True
    return sees


def tree_attention(b, masks, positions, words, window=0, sinks=None):
    """out, lse and the bounds of their errors of a batch (kv_reference.Batch), as kv_reference.attention counts them."""
    dev = b.q.device
    k_pages, v_pages, k_scales, v_scales = b.pages()
    out = torch.zeros(b.T, b.heads, b.dim, dtype=torch.float64, device=dev)
    lse = torch.full((b.T, b.heads), -math.inf, dtype=torch.float64, device=dev)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    words_of, places = masks.cpu().tolist(), positions.cpu().tolist() if positions is not None else [0] * b.T
    for s, full in enumerate(b.kv):
        r0, r1 = b.offsets[s], b.offsets[s + 1]
        held = min(full, b.table.shape[1] * b.page)
        if r1 == r0:
            continue
        sees = seen_by_masks(words_of[r0:r1], places[r0:r1], r1 - r0, full, words, window)[:, :held].to(dev)
        for h in range(b.kv_heads):
            k, here = history(k_pages, k_scales, b.table[s], held, h, b.page)
            v, _ = history(v_pages, v_scales, b.table[s], held, h, b.page)
            seen = sees & here[None]
            k = torch.where(seen.any(0)[:, None], k, 0.0)
            strange = ~torch.isfinite(v)
            vf = torch.where(strange, 0.0, v)
            g = b.heads // b.kv_heads
            for head in range(h * g, (h + 1) * g):
                q = b.q[r0:r1, head].double()
                z = torch.where(seen, (q @ k.T) / math.sqrt(b.dim), -math.inf)
                size = torch.where(seen, (q.abs() @ k.abs().T) / math.sqrt(b.dim), 0.0).nan_to_num(0.0, 0.0, 0.0)
                none = torch.full((r1 - r0,), -math.inf, dtype=torch.float64, device=dev)
                dz = (b.dim + 8) * U * (size.amax(1) if held else 0.0)
                top = z.amax(1) if held else none
                if sinks is not None:
                    top = torch.maximum(top, sinks[head].double())
                top = torch.where(top == -math.inf, 0.0, top)
                w = torch.exp(z - top[:, None])
                total = w.sum(1) + (torch.exp(sinks[head].double() - top) if sinks is not None else 0.0)
                w = torch.where(total[:, None] > 0, w / total[:, None], torch.where(total[:, None] == 0, 0.0, total[:, None]))
                o = torch.where((seen.double() @ strange.double()) > 0, math.nan, w @ vf)
                out[r0:r1, head] = o
                lse[r0:r1, head] = torch.where(total > 0, top + torch.log(total), torch.where(total == 0, none, total))
                rel = 2 * dz + 2 * top.abs() * 4 * U + (held + 64) * U
                stored = EPS[torch.bfloat16] if b.dtype == torch.bfloat16 else 0.0
                tol[r0:r1, head] = EPS[b.dtype] * o.abs() * (1 + 2.0 ** -7) + (rel + stored)[:, None] * (w @ vf.abs()) + 1e-30
                ltol[r0:r1, head] = rel + 8 * U * (1 + top.abs())
    return out, lse, tol, ltol


def weights(b, lse, scores, causal=True, window=0, decay=1.0):
    """The new scores of a batch's cache and the bounds of their errors.

    A weight exp(z - lse) is off by what its exponent is: the product's sum ((dim + 8) half steps of its terms' sizes), the rounded scale and
    the rounded lse and log2(e) (4 half steps of either), and by 4 half steps of its own; the sum by a half step a term at most, in any order."""
    dev = b.q.device
    k_pages, _, k_scales, _ = b.pages()
    new, tol = scores.double().clone(), torch.zeros_like(scores, dtype=torch.float64)
    lse = lse.double()
    g = b.heads // b.kv_heads
    for s, full in enumerate(b.kv):
        r0, r1 = b.offsets[s], b.offsets[s + 1]
        held = min(full, b.table.shape[1] * b.page)
        if r1 == r0 or held == 0:
            continue
        p0 = full - (r1 - r0)
        pos, j = torch.arange(p0, full, device=dev)[:, None], torch.arange(held, device=dev)[None]
        seen = torch.ones(r1 - r0, held, dtype=torch.bool, device=dev)
        if causal:
            seen = seen & (j <= pos)
        if window > 0:
            seen = seen & (j > pos - window)
        for h in range(b.kv_heads):
            k, here = history(k_pages, k_scales, b.table[s], held, h, b.page)
            total, off = torch.zeros(held, dtype=torch.float64, device=dev), torch.zeros(held, dtype=torch.float64, device=dev)
            for head in range(h * g, (h + 1) * g):
                q = b.q[r0:r1, head].double()
                z = (q @ k.T) / math.sqrt(b.dim)
                row = lse[r0:r1, head][:, None]
                w = torch.where(seen & (row != -math.inf), torch.exp(z - row), 0.0)
                size = (q.abs() @ k.abs().T) / math.sqrt(b.dim)
                rel = (b.dim + 8) * U * size + 4 * U * (z.abs() + row.abs()) + 4 * U
                total += w.sum(0)
                off += torch.where(w > 0, w * rel, 0.0).sum(0)
            off += ((r1 - r0) * g + 64) * U * total
            tok = torch.arange(held, device=dev)[here]
            page, slot = b.table[s].long()[tok // b.page], tok % b.page
            old = torch.where(tok < p0, scores[page, h, slot].double() * decay, 0.0) if decay else torch.zeros(len(tok), dtype=torch.float64, device=dev)
            new[page, h, slot] = old + total[here]
            tol[page, h, slot] = off[here] + 3 * U * (old + total[here]).abs() + 1e-37
    return new, tol


def select(scores, lens, table, page, n_pages, budget, first, recent):
    """keep [S, Hk, budget] and keep_lens [S], by a sort of each sequence and head."""
    scores, table = scores.cpu(), table.cpu().long()
    S, hk = len(lens), scores.shape[1]
    keep, kept = torch.full((S, hk, budget), -1, dtype=torch.int32), torch.zeros(S, dtype=torch.int32)
    for s, kv in enumerate(lens):
        held = min(max(kv, 0), table.shape[1] * page)
        j = torch.arange(held)
        ids = table[s][j // page]
        j = j[(ids >= 0) & (ids < n_pages)]
        kept[s] = n = min(budget, len(j))
        for h in range(hk):
            x = scores[table[s][j // page], h, j % page].double()
            x = torch.where(torch.isnan(x), -math.inf, x) + 0.0
            sure = (j < first) | (j >= kv - recent)
            # kept for sure before all others, then the larger score, then the lower token: sorts that keep the order of equals
            order = torch.argsort(-x, stable=True)
            order = order[torch.argsort((~sure[order]).int(), stable=True)]
            keep[s, h, :n] = j[order[:n]].sort().values.int()
    return keep, kept


def compact(tensors, lens, table, page, keep, keep_lens, first):
    """Every tensor [n_pages, Hk, page, ...] with its kept tokens moved."""
    table, got = table.cpu().tolist(), [t.clone() for t in tensors]
    for s in range(len(lens)):
        at = int(first[s]) if first is not None else 0
        for h in range(tensors[0].shape[1]):
            tokens = (keep[s, h] if keep.dim() == 3 else keep[s])[:int(keep_lens[s])].tolist()
            for i, j in enumerate(tokens):
                for t, new in zip(tensors, got):
                    new[table[s][(at + i) // page], h, (at + i) % page] = t[table[s][j // page], h, j % page]
    return got
