"""Writing rows into a paged key/value cache and reading them back, against plain indexing: everything is exact."""
import math

import pytest
import torch

from kv_reference import Batch, history, quantised

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROWS, KV = [1, 0, 7, 33, 1], [1, 5, 7, 70, 300]


def places(b):
    """(row, page, slot) of every row whose token is there."""
    out = []
    for s, n in enumerate(b.rows):
        for i in range(n):
            pos = b.kv[s] - n + i
            if pos >= 0 and pos // b.page < b.table.shape[1]:
                page = int(b.table[s, pos // b.page])
                if 0 <= page < b.k_pages.shape[0]:
                    out.append((b.offsets[s] + i, page, pos % b.page))
    return [torch.tensor(x, device=DEV) for x in zip(*out)]


def check_append(lib, b):
    ctx, pages, batch = b.context(lib)
    want = [x.clone() if x is not None else None for x in b.pages()]
    row, page, slot = places(b)
    for what, x in enumerate((b.k, b.v)):
        if b.fmt == "fp8":
            codes, scales = quantised(x)
            want[what].view(torch.uint8)[page, :, slot] = codes.to(DEV)[row]
            want[2 + what][page, :, slot] = scales.to(DEV)[row]
        else:
            want[what][page, :, slot] = x[row]
    ctx.moe_kv_append(b.k, b.v, pages, batch)
    torch.cuda.synchronize()
    for got, ref, name in zip(b.pages(), want, ("k_pages", "v_pages", "k_scales", "v_scales")):
        if ref is not None:
            assert torch.equal(got.view(torch.uint8), ref.view(torch.uint8)), name


@pytest.mark.parametrize("fmt", ["", "fp8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,page,kv_heads", [(16, 8, 1), (64, 16, 2), (80, 8, 3), (112, 32, 1), (128, 128, 4), (256, 256, 5)])
def test_append_and_gather(gpu_lib, dim, page, kv_heads, dtype, fmt):
    b = Batch(ROWS, KV, 2 * kv_heads, kv_heads, dim, page, dtype, fmt, seed=dim + page)
    check_append(gpu_lib, b)
    ctx, pages, batch = b.context(gpu_lib)
    # outputs with strides of their own
    wide = torch.full((b.T, 3 * kv_heads * dim), 7.0, dtype=dtype, device=DEV)
    k, v = (wide[:, i * kv_heads * dim:(i + 1) * kv_heads * dim].unflatten(1, (kv_heads, dim)) for i in (0, 2))
    ctx.moe_kv_gather(pages, batch, k=k, v=v)
    for got, cache, scales in ((k, b.k_pages, b.k_scales), (v, b.v_pages, b.v_scales)):
        for s, n in enumerate(b.rows):
            for h in range(kv_heads):
                ref = history(cache, scales, b.table[s], b.kv[s], h, page)[0][b.kv[s] - n:]
                assert torch.equal(got[b.offsets[s]:b.offsets[s + 1], h], ref.to(dtype))
    assert (wide[:, kv_heads * dim:2 * kv_heads * dim] == 7.0).all()
    k2, v2 = ctx.moe_kv_gather(pages, batch, T=b.T)
    assert torch.equal(k2, k) and torch.equal(v2, v)


def test_rows_that_are_not_there_are_not_written_and_read_as_zeros(gpu_lib):
    # a page given back, a table too short, an entry past the pages, more rows than tokens, rows past the batch's
    b = Batch([40, 6, 3, 1], [40, 30, 2, 9], 4, 2, 64, 16, dropped=((0, 1),), seed=5)
    b.table[1, 1] = b.k_pages.shape[0]
    b.table = b.table[:, :2].contiguous()
    check_append(gpu_lib, b)
    ctx, pages, batch = b.context(gpu_lib)
    k, v = ctx.moe_kv_gather(pages, batch, T=b.T + 2)[0:2]
    there = torch.zeros(b.T + 2, dtype=torch.bool, device=DEV)
    there[places(b)[0]] = True
    assert not there[16:32].any() and not there[40:46].any() and not there[46] and not there[b.T:].any()
    for got, ref in ((k, b.k), (v, b.v)):
        assert torch.equal(got[:b.T][there[:b.T]], ref[there[:b.T]]) and (got[~there] == 0).all()


def test_rows_at_the_edges_of_the_codes(gpu_lib):
    b = Batch([12], [12], 2, 2, 64, 16, torch.float32, "fp8", seed=6)
    x = torch.randn(12, 2, 64, generator=torch.Generator().manual_seed(1))
    x[0] = 0
    x[1] *= 448.0 / x[1].abs().max()                     # the largest code
    x[2] *= 448.0 * (1 + 2.0 ** -23) / x[2].abs().max()
    x[3] *= 1e-36                                        # the smallest scale
    x[4] *= 2.0 ** -140                                  # below the normal numbers
    x[5, :, 3] = math.nan
    x[6, 0, 63] = math.inf
    x[7, 1, 0] = -math.inf
    x[8] *= 3.4e38 / x[8].abs().max()
    x[9] = 2.0 ** -9 * torch.arange(64) - 0.06           # ties of the codes' rounding
    x[9, :, 0] = 1.0
    b.k.copy_(x)
    b.v.copy_(-x)
    check_append(gpu_lib, b)


@pytest.mark.parametrize("n_seqs", [1, 64, 65, 300, 4100])
def test_many_sequences(gpu_lib, n_seqs):
    rows = [(s * 7) % 3 for s in range(n_seqs)]
    rows[-1] = 2
    kv = [n + (s * 13) % 40 for s, n in enumerate(rows)]
    check_append(gpu_lib, Batch(rows, kv, 1, 1, 16, 8, seed=n_seqs))


def test_many_empty_sequences_between_two_rows(gpu_lib):
    rows = [1] + [0] * 70 + [2] + [0] * 200 + [1, 0, 3]
    check_append(gpu_lib, Batch(rows, [n + 3 for n in rows], 2, 2, 64, 8, seed=3))


def test_pages_far_into_a_cache(gpu_lib):
    # rows past 2^32 bytes of the pages
    n_pages, page, kv_heads, dim = 150000, 16, 8, 128
    b = Batch([3, 2], [20, 17], 8, kv_heads, dim, page, seed=9)
    ids = b.table.clone()
    b.k_pages, b.v_pages = (torch.empty(n_pages, kv_heads, page, dim, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    b.table = torch.where(ids >= 0, n_pages - 1 - ids, -1).to(torch.int32)
    ctx, pages, batch = b.context(gpu_lib)
    ctx.moe_kv_append(b.k, b.v, pages, batch)
    row, at, slot = places(b)
    assert torch.equal(b.k_pages[at, :, slot], b.k[row]) and torch.equal(b.v_pages[at, :, slot], b.v[row])
    k, v = ctx.moe_kv_gather(pages, batch, T=b.T)
    assert torch.equal(k, b.k) and torch.equal(v, b.v)
