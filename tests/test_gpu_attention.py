"""Attention over a paged cache against the definition in 64 bits.  Bounds count the roundings: of the stored result, of the bf16
weights, of fp32 scores, exponentials and sums (kv_reference.attention)."""
import math

import pytest
import torch

from kv_reference import Batch, assert_within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def check(lib, b, causal=True, window=0, sinks=None, strided=False):
    ctx, pages, batch = b.context(lib)
    lse = torch.full((b.T, b.heads), 7.0, device=DEV)
    out = torch.full((b.T, b.heads, b.dim), 7.0, dtype=b.dtype, device=DEV)
    if strided:
        wide = torch.full((b.T, (b.heads + 1) * b.dim), 7.0, dtype=b.dtype, device=DEV)
        out = wide[:, b.dim:].unflatten(1, (b.heads, b.dim))
    ctx.moe_paged_attention(b.q, pages, batch, causal=causal, window=window, sinks=sinks, out=out, lse=lse)
    ref, ref_lse, tol, ltol = b.reference(causal, window, sinks)
    assert_within(out, ref, tol, "out")
    assert_within(lse, ref_lse, ltol, "lse")
    if strided:
        assert (wide[:, :b.dim] == 7.0).all()
    return out, lse


def sinks_of(heads, seed=3):
    return torch.randn(heads, generator=torch.Generator().manual_seed(seed)).to(DEV)


ROWS, KV = [1, 0, 4, 40, 1, 130], [1, 9, 4, 75, 300, 131]


@pytest.mark.parametrize("fmt", ["", "fp8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,page,kv_heads,group", [(16, 8, 1, 1), (32, 16, 2, 4), (64, 32, 2, 8), (80, 8, 1, 5), (96, 64, 2, 2),
                                                     (112, 16, 1, 7), (128, 16, 2, 8), (128, 128, 1, 16), (256, 8, 1, 4), (208, 32, 2, 3)])
def test_types_and_layouts(gpu_lib, dim, page, kv_heads, group, dtype, fmt):
    b = Batch(ROWS, KV, kv_heads * group, kv_heads, dim, page, dtype, fmt, seed=dim + group)
    check(gpu_lib, b, strided=True)
    check(gpu_lib, b, window=50, sinks=sinks_of(b.heads))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 8, 33, 128, 2 ** 29])
@pytest.mark.parametrize("dtype,fmt,dim", [(torch.bfloat16, "", 64), (torch.bfloat16, "fp8", 128), (torch.float32, "", 64), (torch.bfloat16, "", 128)])
def test_masks(gpu_lib, causal, window, dtype, fmt, dim):
    b = Batch([1, 3, 64, 20, 97, 300], [5, 3, 64, 150, 230, 1000], 8, 2, dim, 16, dtype, fmt, seed=window % 97)
    check(gpu_lib, b, causal, window, sinks_of(8) if window % 2 else None)


@pytest.mark.parametrize("kv", [1, 2, 31, 32, 33, 127, 128, 129, 255, 257, 500, 1024, 1025, 4097, 20000])
@pytest.mark.parametrize("dtype,fmt", [(torch.bfloat16, ""), (torch.bfloat16, "fp8"), (torch.float32, "")])
def test_single_tokens_at_every_length(gpu_lib, kv, dtype, fmt):
    check(gpu_lib, Batch([1], [kv], 8, 2, 128, 16, dtype, fmt, seed=kv), sinks=sinks_of(8) if kv % 2 else None)


@pytest.mark.parametrize("rows", [2, 3, 5, 9, 17, 32, 33, 63, 64, 65, 127, 128, 129, 257])
@pytest.mark.parametrize("group", [1, 5, 8])
def test_rows_at_the_edges_of_tiles(gpu_lib, rows, group):
    check(gpu_lib, Batch([rows, 1, rows], [rows + 77, 9, rows], 2 * group, 2, 64, 16, seed=rows))
    check(gpu_lib, Batch([rows, 1], [rows + 600, 40], group, 1, 128, 16, fmt="fp8", seed=rows))


@pytest.mark.parametrize("dtype,fmt", [(torch.bfloat16, ""), (torch.bfloat16, "fp8"), (torch.float32, "fp8")])
def test_rows_that_see_nothing(gpu_lib, dtype, fmt):
    # no tokens at all; fewer tokens than rows; every page given back; a window all of whose pages are gone; a hole in the middle
    b = Batch([2, 5, 1, 2, 3], [0, 2, 40, 100, 90], 4, 2, 64, 16, dtype, fmt, seed=11,
              dropped=((2, 0), (2, 1), (2, 2), (3, 5), (3, 6), (4, 2), (4, 3)))
    out, lse = check(gpu_lib, b, window=20)
    assert (out[:2] == 0).all() and (lse[:2] == -math.inf).all() and (out[2:5] == 0).all() and (out[7] == 0).all()
    assert (lse[7] == -math.inf).all()
    s = sinks_of(4)
    out, lse = check(gpu_lib, b, window=20, sinks=s)
    assert (out[:2] == 0).all() and torch.allclose(lse[:2], s.expand(2, 4), rtol=1e-6, atol=1e-6)
    s[1] = -math.inf
    check(gpu_lib, b, sinks=s)
    check(gpu_lib, b, causal=False)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("rows,dim,group", [(4, 64, 4), (30, 128, 1), (150, 128, 8), (150, 64, 8)])
@pytest.mark.parametrize("dtype,fmt", [(torch.bfloat16, ""), (torch.bfloat16, "fp8"), (torch.float32, ""), (torch.float32, "fp8")])
def test_strange_values_reach_only_the_rows_that_see_them(gpu_lib, dtype, fmt, rows, dim, group, bad):
    kv = rows + 100
    b = Batch([rows, 1], [kv, 50], group, 1, dim, 16, dtype, fmt, seed=13)
    at = kv - rows + rows // 2            # token of the middle row
    page, slot = int(b.table[0, at // 16]), at % 16
    for cache, scales in ((b.v_pages, b.v_scales), (b.k_pages, b.k_scales)):
        keep = cache.clone(), scales.clone() if scales is not None else None
        if fmt == "fp8" and bad != math.inf:
            scales[page, 0, slot] = 255
        elif fmt == "fp8":
            cache.view(torch.uint8)[page, 0, slot, 5] = 0xff
        else:
            cache[page, 0, slot, 5] = bad
        ctx, pages, batch = b.context(gpu_lib)
        out = ctx.moe_paged_attention(b.q, pages, batch)
        ref, _, tol, _ = b.reference()
        sees = torch.arange(b.T, device=DEV) >= rows // 2
        sees[rows:] = False
        assert_within(out[~sees], ref[~sees], tol[~sees])
        if cache is b.v_pages:
            assert not torch.isfinite(out[sees][..., 5].float()).any()
            others = [d for d in range(dim) if d != 5]
            if not (fmt == "fp8" and bad != math.inf):
                assert torch.isfinite(out[sees][..., others].float()).all()
                if fmt == "":
                    want = torch.full_like(out[sees][..., 5].float(), bad)
                    assert torch.equal(out[sees][..., 5].float().nan_to_num(123.0, 1e30, -1e30), want.nan_to_num(123.0, 1e30, -1e30))
        elif math.isnan(bad) or fmt == "fp8":
            assert not torch.isfinite(out[sees].float()).any()
        cache.copy_(keep[0])
        if scales is not None:
            scales.copy_(keep[1])


def test_large_and_small_scores(gpu_lib):
    # maxima that keep growing along the history, then fall; scores far apart
    for dtype in (torch.bfloat16, torch.float32):
        b = Batch([1, 6, 200], [900, 700, 500], 8, 2, 64, 16, dtype, seed=17)
        for s in range(3):
            for i in range(-(-b.kv[s] // 16)):
                if int(b.table[s, i]) >= 0:
                    b.k_pages[int(b.table[s, i])] *= (1 + i if s != 1 else 40 - i) * 0.5
        check(gpu_lib, b)
        check(gpu_lib, b, window=100, sinks=100 * sinks_of(8))


@pytest.mark.parametrize("n_seqs", [63, 64, 65, 255, 257, 700])
def test_many_sequences(gpu_lib, n_seqs):
    rows = [[1, 1, 0, 1, 5][s % 5] for s in range(n_seqs)]
    kv = [max(n, (s * 37) % 200) for s, n in enumerate(rows)]
    kv[n_seqs // 2] = 3000
    check(gpu_lib, Batch(rows, kv, 4, 1, 64, 16, seed=n_seqs))


def test_work_that_needs_every_unit_of_the_partial_results(gpu_lib):
    # long histories under few rows, more than the workspace holds pieces for
    b = Batch([33] * 40, [700] * 40, 8, 8, 64, 16, seed=19)
    check(gpu_lib, b)
    b = Batch([4] * 24 + [1] * 30, [2500] * 24 + [1500] * 30, 16, 4, 64, 16, fmt="fp8", seed=20)
    check(gpu_lib, b)


def test_pages_far_into_a_cache(gpu_lib):
    # the tokens' rows lie past 2^32 bytes of the pages
    n_pages, page, kv_heads, dim = 150000, 16, 8, 128
    b = Batch([1, 40], [200, 170], 16, kv_heads, dim, page, seed=23)
    small_k, small_v, ids = b.k_pages, b.v_pages, b.table.clone()
    n = small_k.shape[0]
    b.k_pages, b.v_pages = (torch.empty(n_pages, kv_heads, page, dim, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    b.k_pages[-n:], b.v_pages[-n:] = small_k, small_v
    b.table = torch.where(ids >= 0, ids + (n_pages - n), -1).to(torch.int32)
    check(gpu_lib, b)


def test_bad_descriptors_give_no_wild_accesses(gpu_lib):
    """Offsets that descend, lengths past the table, entries past the pages: results mean nothing, but nothing outside the
    caller's tensors is touched (the host bounds every index by what it knows: T, the table's shape, the pages' number)."""
    b = Batch([3, 3, 60], [30, 30, 100], 8, 2, 64, 16, seed=29)
    ctx, pages, batch = b.context(gpu_lib)
    guard = torch.full((b.T + 2, 8, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    out = guard[1:-1]
    for off, lens in (([0, 50, 3, 66], [30, 30, 100]), ([-5, 3, 6, 10 ** 9], [30, 2 ** 31 - 1, 100]), ([0, 3, 6, 66], [-7, -2 ** 31, 5])):
        b.row_offsets.copy_(torch.tensor(off, dtype=torch.int32))
        b.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        ctx.moe_paged_attention(b.q, pages, batch, out=out)
        ctx.moe_kv_gather(pages, batch, T=b.T)
        torch.cuda.synchronize()
        assert (guard[0] == 7.0).all() and (guard[-1] == 7.0).all()


def test_lse_joins_two_parts_of_a_history(gpu_lib):
    """Attention to the first 96 tokens and to the rest, joined by their log-sum-exp, is attention to all."""
    b = Batch([5], [230], 8, 2, 64, 16, torch.float32, seed=31)
    whole, _ = check(gpu_lib, b)
    first = Batch([5], [96], 8, 2, 64, 16, torch.float32, seed=31)
    first.q, first.k_pages, first.v_pages, first.table = b.q, b.k_pages, b.v_pages, b.table
    o1, l1 = check(gpu_lib, first, causal=False)
    rest = b.table.clone()
    rest[0, :6] = -1
    keep, b.table = b.table, rest
    o2, l2 = check(gpu_lib, b)
    m = torch.maximum(l1, l2)
    w1, w2 = torch.exp(l1 - m), torch.exp(l2 - m)
    joined = (o1 * w1[..., None] + o2 * w2[..., None]) / (w1 + w2)[..., None]
    assert torch.allclose(joined, whole, rtol=1e-5, atol=1e-5)
    b.table = keep


def test_same_bits_again_and_on_another_stream(gpu_lib):
    b = Batch([1, 4, 130, 1], [3000, 900, 700, 5000], 8, 2, 128, 16, seed=37)
    ctx, pages, batch = b.context(gpu_lib)
    ref = ctx.moe_paged_attention(b.q, pages, batch)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [ctx.moe_paged_attention(b.q, pages, batch) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for x in again:
        assert torch.equal(x, ref)


def test_replays_of_a_graph_take_the_descriptors_as_they_are(gpu_lib):
    """Append, attention and gather are captured once; lengths, rows and values change between the replays."""
    b = Batch([1, 3, 1, 40], [500, 300, 2000, 90], 8, 2, 64, 16, fmt="fp8", seed=41)
    b.table = torch.arange(4 * 200, dtype=torch.int32, device=DEV).view(4, 200)
    b.k_pages, b.v_pages = (torch.zeros(800, 2, 16, 64, device=DEV).to(torch.float8_e4m3fn) for _ in range(2))
    b.k_scales, b.v_scales = (torch.full((800, 2, 16), 127, dtype=torch.uint8, device=DEV) for _ in range(2))
    ctx, pages, batch = b.context(gpu_lib)
    out, k, v = torch.empty_like(b.q.contiguous()), torch.empty_like(b.k.contiguous()), torch.empty_like(b.v.contiguous())

    def step(out, k, v):
        ctx.moe_kv_append(b.k, b.v, pages, batch)
        ctx.moe_paged_attention(b.q, pages, batch, out=out)
        ctx.moe_kv_gather(pages, batch, k=k, v=v)

    step(out, k, v)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, k, v)
    for rep in range(4):
        gen = torch.Generator().manual_seed(rep)
        b.q.copy_(torch.randn(b.q.shape, generator=gen))
        b.k.copy_(torch.randn(b.k.shape, generator=gen))
        b.v.copy_(torch.randn(b.v.shape, generator=gen))
        cut = sorted(torch.randint(0, b.T + 1, (3,), generator=gen).tolist())
        b.offsets = [0] + cut + [b.T]
        b.kv = [b.offsets[s + 1] - b.offsets[s] + int(torch.randint(0, 3000, (1,), generator=gen)) for s in range(4)]
        b.row_offsets.copy_(torch.tensor(b.offsets, dtype=torch.int32))
        b.kv_lens.copy_(torch.tensor(b.kv, dtype=torch.int32))
        eager = [torch.empty_like(x) for x in (out, k, v)]
        step(*eager)
        torch.cuda.synchronize()
        for x in (out, k, v):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip((out, k, v), eager):
            assert torch.equal(got, want), f"replay {rep}"
        ref, _, tol, _ = b.reference()
        assert_within(out, ref, tol, f"replay {rep}")


@pytest.mark.parametrize("n_seqs", [50, 200, 400])
def test_prompts_among_many_sequences(gpu_lib, n_seqs):
    rows = [[1, 0, 2, 1][s % 4] for s in range(n_seqs)]
    kv = [max(n, (s * 29) % 150) for s, n in enumerate(rows)]
    for s, n, k in ((3, 90, 700), (n_seqs - 2, 300, 300), (n_seqs // 2, 17, 2500)):
        rows[s], kv[s] = n, k
    check(gpu_lib, Batch(rows, kv, 16, 2, 64, 16, seed=n_seqs), sinks=sinks_of(16))


@pytest.mark.parametrize("dim", [64, 80, 128, 256])
@pytest.mark.parametrize("dtype,fmt", [(torch.bfloat16, ""), (torch.bfloat16, "fp8"), (torch.float32, "")])
def test_long_histories_in_several_pieces(gpu_lib, dim, dtype, fmt):
    check(gpu_lib, Batch([70, 3, 1, 20], [4100, 3000, 5000, 1700], 8, 2, dim, 32, dtype, fmt, seed=dim), sinks=sinks_of(8))
    check(gpu_lib, Batch([150], [3333], 4, 2, dim, 8, dtype, fmt, seed=dim + 1), window=1500)


def test_a_first_call_may_be_captured(gpu_lib):
    """What a context clears once belongs to the graph then, and eager calls before and between its replays find it cleared too."""
    b = Batch([1, 40], [3000, 2000], 8, 2, 64, 16, seed=43)
    ref, _, tol, _ = b.reference()
    ctx, pages, batch = b.context(gpu_lib)
    ctx.workspace.fill_(0xff)
    out = torch.zeros(b.T, 8, 64, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.moe_paged_attention(b.q, pages, batch, out=out)
    for _ in range(3):
        assert_within(ctx.moe_paged_attention(b.q, pages, batch), ref, tol, "eager")
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert_within(out, ref, tol, "replay")
