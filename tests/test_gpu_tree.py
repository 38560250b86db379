"""Trees of drafted tokens: masks and positions exactly, attention against the definition in 64 bits (bounds: keep_reference.tree_attention)."""
import ctypes
import math
import random

import pytest
import torch

import keep_reference as ref
from kv_reference import Batch, assert_within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def parents_of(rows, kind, seed=0):
    """Parents of every sequence's rows: a chain, a star, a tree with one root, several with many, or numbers that name no earlier row too."""
    r, got = random.Random(seed), []
    for n in rows:
        for i in range(n):
            got.append({"chain": i - 1, "star": 0 if i else -1, "tree": r.randint(i // 3, i - 1) if i else -1, "forest": r.randint(-1, i - 1),
                        "wild": r.choice([r.randint(-1, max(0, i - 1)), i, n + 3, -7, 2 ** 31 - 1, -2 ** 31])}[kind])
    return got


def masks_of(b, parents, words, window):
    masks, positions = ref.tree_masks(parents, b.offsets, b.kv, words, window)
    return masks.to(b.device), positions.to(b.device)


@pytest.mark.parametrize("kind", ["chain", "star", "tree", "forest", "wild"])
@pytest.mark.parametrize("words,rows", [(1, [1, 0, 2, 63, 64, 65, 8]), (2, [128, 129, 65, 1, 300]), (3, [192, 193, 7, 130]), (4, [256, 200, 33, 1000]),
                                        (7, [448, 449, 5]), (16, [1024, 1025, 1, 700])])
@pytest.mark.parametrize("window", [0, 1, 2, 70, 500])
def test_masks(gpu_lib, kind, words, rows, window):
    kv = [n + 37 * s for s, n in enumerate(rows)]
    kv[0], kv[-1] = 0, max(0, rows[-1] - 3)              # fewer tokens than rows
    offsets = [0]
    for n in rows:
        offsets.append(offsets[-1] + n)
    parents = parents_of(rows, kind, words + window)
    T = len(parents) + 5                                 # (rows of no sequence)
    ctx = gpu_lib.KVContext(2, 1, 32, 16, torch.float32, device=DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    batch = ctx.pack_batch(torch.tensor(offsets, **i32), torch.tensor(kv, **i32), torch.zeros(len(rows), 1, **i32))
    masks, positions = torch.full((T, words), 77, dtype=torch.int64, device=DEV), torch.full((T,), 77, **i32)
    ctx.moe_tree_masks(torch.tensor(parents + [3] * 5, **i32), batch, words=words, window=window, masks=masks, positions=positions)
    want, places = ref.tree_masks(parents, offsets, kv, words, window)
    assert torch.equal(masks[:-5].cpu(), want) and torch.equal(positions[:-5].cpu(), places)
    assert (masks[-5:] == 77).all() and (positions[-5:] == 77).all()


def test_masks_alone_and_bad_offsets(gpu_lib):
    """Without positions; sequences whose offsets descend or leave the batch are left as they were; many slots."""
    ctx = gpu_lib.KVContext(2, 1, 32, 16, torch.float32, device=DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    parents = torch.tensor(parents_of([6, 6], "tree"), **i32)
    for offsets in ([0, 6, 12], [0, 6, 13], [0, 6, 2], [-4, 6, 12]):
        batch = ctx.pack_batch(torch.tensor(offsets, **i32), torch.tensor([6, 9], **i32), torch.zeros(2, 1, **i32))
        masks = torch.full((12, 1), 77, dtype=torch.int64, device=DEV)
        ctx._call("moe_tree_masks", parents.data_ptr(), 12, batch, 1, 0, masks.data_ptr(), None)
        want = ref.tree_masks(parents.tolist(), [0, 6, 12], [6, 9], 1, 0)[0]
        for s in range(2):
            legal = 0 <= offsets[s] <= offsets[s + 1] <= 12
            assert torch.equal(masks[6 * s:6 * s + 6].cpu(), want[6 * s:6 * s + 6] if legal else torch.full((6, 1), 77))
    S = 5000
    rows = [3 if s % 1000 == 7 else 0 for s in range(S)]
    off = torch.tensor([0] + rows).cumsum(0)
    parents = parents_of(rows, "tree")
    batch = ctx.pack_batch(off.to(**i32), torch.full((S,), 9, **i32), torch.zeros(S, 1, **i32))
    masks, _ = ctx.moe_tree_masks(torch.tensor(parents, **i32), batch)
    assert torch.equal(masks.cpu(), ref.tree_masks(parents, off.tolist(), [9] * S, 1, 0)[0])


def check(lib, b, masks, positions=None, window=0, sinks=None, strided=False):
    ctx, pages, batch = b.context(lib)
    lse = torch.full((b.T, b.heads), 7.0, device=DEV)
    out = torch.full((b.T, b.heads, b.dim), 7.0, dtype=b.dtype, device=DEV)
    if strided:
        wide = torch.full((b.T, (b.heads + 1) * b.dim), 7.0, dtype=b.dtype, device=DEV)
        out = wide[:, b.dim:].unflatten(1, (b.heads, b.dim))
    ctx.moe_tree_attention(b.q, pages, batch, masks, positions=positions, window=window, sinks=sinks, out=out, lse=lse)
    want, want_lse, tol, ltol = ref.tree_attention(b, masks, positions, masks.shape[1], window, sinks)
    assert_within(out, want, tol, "out")
    assert_within(lse, want_lse, ltol, "lse")
    if strided:
        assert (wide[:, :b.dim] == 7.0).all()
    return out, lse


def sinks_of(heads, seed=3):
    return torch.randn(heads, generator=torch.Generator().manual_seed(seed)).to(DEV)


@pytest.mark.parametrize("fmt", ["", "fp8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,page,kv_heads,group", [(16, 8, 1, 1), (32, 16, 2, 4), (64, 32, 2, 8), (80, 8, 1, 5), (112, 16, 1, 7), (128, 16, 2, 8),
                                                     (128, 128, 1, 16), (256, 8, 1, 4), (208, 32, 2, 3)])
def test_types_and_layouts(gpu_lib, dim, page, kv_heads, group, dtype, fmt):
    rows, kv = [1, 0, 4, 40, 64, 130], [1, 9, 4, 75, 300, 131]
    b = Batch(rows, kv, kv_heads * group, kv_heads, dim, page, dtype, fmt, seed=dim + group)
    check(gpu_lib, b, *masks_of(b, parents_of(rows, "tree", dim), 1, 0), strided=True)
    check(gpu_lib, b, *masks_of(b, parents_of(rows, "forest", dim), 3, 50), window=50, sinks=sinks_of(b.heads))


@pytest.mark.parametrize("words", [1, 2, 4, 5, 16])
@pytest.mark.parametrize("window", [0, 1, 3, 60, 2 ** 29])
@pytest.mark.parametrize("dtype,fmt,dim", [(torch.bfloat16, "", 64), (torch.bfloat16, "fp8", 128), (torch.float32, "", 64)])
def test_words_and_windows(gpu_lib, words, window, dtype, fmt, dim):
    rows = [1, 3, 64, 65, 127, 300]
    kv = [500, 3, 64, 150, 131, 420]
    b = Batch(rows, kv, 8, 2, dim, 16, dtype, fmt, seed=window % 97)
    check(gpu_lib, b, *masks_of(b, parents_of(rows, "tree", words), words, window), window=window, sinks=sinks_of(8) if window % 2 else None)


@pytest.mark.parametrize("start", list(range(0, 34)) + [63, 64, 65, 127, 1000, 4097])
@pytest.mark.parametrize("dtype,fmt", [(torch.bfloat16, ""), (torch.bfloat16, "fp8"), (torch.float32, "")])
def test_trees_behind_every_number_of_tokens(gpu_lib, start, dtype, fmt):
    """Where a tree begins within a step and a page; drafts of one row, and of 16-row and of 128-row tiles."""
    rows = [1, 5, 33, 61, 90]
    b = Batch(rows, [start + n for n in rows], 8, 2, 128, 8, dtype, fmt, seed=start)
    check(gpu_lib, b, *masks_of(b, parents_of(rows, "tree", start), 2, 0))


@pytest.mark.parametrize("dtype,fmt,group", [(torch.bfloat16, "", 8), (torch.bfloat16, "fp8", 2), (torch.float32, "", 4)])
def test_long_histories_in_pieces(gpu_lib, dtype, fmt, group):
    rows = [12, 64, 1]
    b = Batch(rows, [30000, 9000, 5000], 2 * group, 2, 64, 64, dtype, fmt, seed=5)
    check(gpu_lib, b, *masks_of(b, parents_of(rows, "tree", 5), 1, 0))
    check(gpu_lib, b, *masks_of(b, parents_of(rows, "tree", 6), 1, 700), window=700, sinks=sinks_of(b.heads))


def test_a_chain_is_causal(gpu_lib):
    rows, kv = [5, 64, 1, 40, 200], [100, 64, 30, 3000, 900]
    for dtype in (torch.bfloat16, torch.float32):
        b = Batch(rows, kv, 8, 2, 64, 16, dtype, seed=2)
        ctx, pages, batch = b.context(gpu_lib)
        for window in (0, 25):
            masks, positions = masks_of(b, parents_of(rows, "chain"), 1, window)
            out = ctx.moe_tree_attention(b.q, pages, batch, masks, positions=positions, window=window)
            want, _, tol, _ = b.reference(True, window)
            assert_within(out, want, tol)


def test_masks_that_no_tree_gives(gpu_lib):
    """Empty masks, rows that see others but not themselves, later rows, bits past the sequence's rows, positions that are none."""
    rows, kv = [6, 64, 70, 3], [6, 100, 400, 2]
    for dtype, fmt in ((torch.bfloat16, ""), (torch.float32, ""), (torch.bfloat16, "fp8")):
        b = Batch(rows, kv, 4, 2, 64, 16, dtype, fmt, seed=7)
        g = torch.Generator().manual_seed(1)
        masks = torch.randint(-2 ** 63, 2 ** 63 - 1, (b.T, 2), generator=g).to(DEV)
        masks[::5] = 0
        masks[-1] = -1
        out, lse = check(gpu_lib, b, masks)
        assert (out[0] == 0).all() and (lse[0] == -math.inf).all()      # nothing cached, an empty mask
        positions = torch.randint(-2 ** 31, 2 ** 31 - 1, (b.T,), generator=g, dtype=torch.int32).to(DEV)
        check(gpu_lib, b, masks, positions, window=40, sinks=sinks_of(4))


def test_missing_pages_and_short_tables(gpu_lib):
    rows = [4, 20, 9, 64]
    b = Batch(rows, [100, 90, 70, 500], 8, 2, 64, 16, seed=4, dropped=((0, 6), (1, 0), (1, 5), (2, 4), (3, 29), (3, 31)))
    check(gpu_lib, b, *masks_of(b, parents_of(rows, "tree"), 1, 0))
    b.table = b.table[:, :5].contiguous()                # ends before the trees do, or in them
    check(gpu_lib, b, *masks_of(b, parents_of(rows, "tree"), 1, 0))
    check(gpu_lib, b, *masks_of(b, parents_of(rows, "tree"), 1, 30), window=30)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("rows,dim,group", [(4, 64, 4), (30, 128, 1), (60, 128, 8), (60, 64, 8)])
@pytest.mark.parametrize("dtype,fmt", [(torch.bfloat16, ""), (torch.bfloat16, "fp8"), (torch.float32, "")])
def test_strange_values_reach_only_the_rows_that_see_them(gpu_lib, dtype, fmt, rows, dim, group, bad):
    kv = rows + 100
    b = Batch([rows, 1], [kv, 50], group, 1, dim, 16, dtype, fmt, seed=13)
    at = kv - rows + rows // 2                           # token of the middle row
    page, slot = int(b.table[0, at // 16]), at % 16
    masks, positions = masks_of(b, parents_of([rows, 1], "tree", 9), 1, 0)
    sees = ((masks[:, 0] >> (rows // 2)) & 1).bool()
    sees[rows:] = False
    assert sees.any() and not sees.all()
    for what in ("v", "k"):
        pages, scales = (b.v_pages, b.v_scales) if what == "v" else (b.k_pages, b.k_scales)
        keep = pages.clone(), scales.clone() if scales is not None else None
        if fmt == "fp8":
            scales[page, 0, slot] = 255
        else:
            pages[page, 0, slot, 5] = bad
        ctx, packed, batch = b.context(gpu_lib)
        out = ctx.moe_tree_attention(b.q, packed, batch, masks)
        want, _, tol, _ = ref.tree_attention(b, masks, positions, 1)
        assert_within(out[~sees], want[~sees], tol[~sees])
        if what == "v":
            assert not torch.isfinite(out[sees][..., 5].float()).any()
        elif math.isnan(bad) or fmt == "fp8":
            assert not torch.isfinite(out[sees].float()).any()
        pages.copy_(keep[0])
        if scales is not None:
            scales.copy_(keep[1])
