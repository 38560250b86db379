"""Attention over a paged cache where descriptors and contents are at their edges, against the definition in 64 bits (bounds as in
test_gpu_attention.py)."""
import math

import pytest
import torch

from kv_reference import Batch, assert_within, attention

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FORMS = [(torch.bfloat16, ""), (torch.bfloat16, "fp8"), (torch.float32, ""), (torch.float32, "fp8")]


def sinks_of(heads, seed=3):
    return torch.randn(heads, generator=torch.Generator().manual_seed(seed)).to(DEV)


def call(lib, b, **options):
    ctx, pages, batch = b.context(lib)
    lse = torch.full((b.T, b.heads), 7.0, device=DEV)
    out = ctx.moe_paged_attention(b.q, pages, batch, lse=lse, **options)
    return out, lse


def check(lib, b, causal=True, window=0, sinks=None):
    """The reference takes positions from its lengths only where its table reaches that far: entries of -1 take the table there."""
    wide = torch.full((len(b.kv), max(-(-k // b.page) for k in b.kv) + 1), -1, dtype=torch.int32, device=DEV)
    n = min(wide.shape[1], b.table.shape[1])
    wide[:, :n] = b.table[:, :n]
    out, lse = call(lib, b, causal=causal, window=window, sinks=sinks)
    ref, ref_lse, tol, ltol = attention(b.q, b.pages(), b.offsets, b.kv, wide, b.page, causal, window, sinks)
    tol = torch.where(ref.isnan(), 0.0, tol)      # (where the result has no finite value only that is asked for)
    assert_within(out, ref, tol, "out")
    assert_within(lse, ref_lse, ltol, "lse")
    return out, lse


# ---- lengths past the table: the rows keep their positions, the tokens that the table does not reach are not there ----

def short_table(rows, kv, columns, heads, kv_heads, dim, page, dtype, fmt, seed):
    b = Batch(rows, kv, heads, kv_heads, dim, page, dtype, fmt, seed=seed)
    b.table = b.table[:, :columns].contiguous()
    return b


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 5, 40, 2 ** 29])
@pytest.mark.parametrize("dtype,fmt", FORMS)
def test_lengths_past_the_table(gpu_lib, dtype, fmt, window, causal):
    # two pages of eight: positions 12 to 19 and 0 to 39, of which tokens 0 to 15 are there; decode rows inside and far behind
    check(gpu_lib, short_table([8, 40, 1, 1, 3], [20, 40, 16, 200, 9], 2, 4, 2, 64, 8, dtype, fmt, 3), causal, window)
    # decode rows alone; rows for tiles of 32 and of 128
    check(gpu_lib, short_table([1, 1, 1], [70, 64, 50], 4, 8, 1, 128, 16, dtype, fmt, 5), causal, window, sinks_of(8))
    check(gpu_lib, short_table([30, 150, 150], [90, 150, 400], 5, 1, 1, 64, 16, dtype, fmt, 7), causal, window)
    # histories in several pieces
    check(gpu_lib, short_table([2, 140], [6000, 5000], 250, 2, 2, 64, 16, dtype, fmt, 9), causal, window)


@pytest.mark.parametrize("dtype,fmt", FORMS)
@pytest.mark.parametrize("rows", [1, 20, 150])
def test_the_longest_lengths(gpu_lib, rows, dtype, fmt):
    b = Batch([rows, 1], [160, 30], 4, 2, 64, 16, dtype, fmt, seed=rows)
    want, want_lse = call(gpu_lib, b, causal=False)
    b.kv_lens[0] = 2 ** 31 - 1                # every token that the table holds is behind the rows
    for causal in (True, False):
        out, lse = call(gpu_lib, b, causal=causal)
        assert torch.equal(out[:rows], want[:rows]) and torch.equal(lse[:rows], want_lse[:rows])
        for window in (1, 50, 2 ** 30):
            out, lse = call(gpu_lib, b, causal=causal, window=window)
            assert (out[:rows] == 0).all() and (lse[:rows] == -math.inf).all()
            assert torch.isfinite(out.float()).all()


# ---- values that are not finite, where a row first sees anything ----

@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("rows,kv,window,at", [(150, 150, 0, 10), (150, 150, 0, 0), (150, 1000, 200, 700), (150, 1000, 70, 900), (40, 40, 0, 10),
                                               (20, 20, 0, 10), (1, 90, 20, 75)])
@pytest.mark.parametrize("dtype,dim,group", [(torch.bfloat16, 64, 1), (torch.bfloat16, 128, 8), (torch.bfloat16, 256, 1), (torch.bfloat16, 80, 2),
                                             (torch.float32, 64, 1)])
def test_strange_values_in_a_first_step(gpu_lib, dtype, dim, group, rows, kv, window, at, bad):
    b = Batch([rows], [kv], group, 1, dim, 16, dtype, seed=13)
    b.v_pages[int(b.table[0, at // 16]), 0, at % 16, 5] = bad
    out, lse = check(gpu_lib, b, window=window)
    pos = torch.arange(kv - rows, kv, device=DEV)
    sees = (pos >= at) & ((pos - at < window) if window else torch.ones_like(pos, dtype=torch.bool))
    assert sees.any()
    got = out[sees][..., 5].float()
    assert torch.equal(got.nan_to_num(123.0, 1e30, -1e30), torch.full_like(got, bad).nan_to_num(123.0, 1e30, -1e30))
    assert torch.isfinite(out[~sees].float()).all() and torch.isfinite(lse).all()
    others = [d for d in range(dim) if d != 5]
    assert torch.isfinite(out[..., others].float()).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,group", [(1, 4), (4, 8), (30, 1), (150, 1)])
@pytest.mark.parametrize("dim", [16, 48, 64, 80, 96, 112, 128, 144, 208, 256])
def test_keys_of_minus_infinity_are_weights_of_zero(gpu_lib, dim, rows, group, dtype):
    """At every width, in the first dimensions too: a score of minus infinity, not NaN."""
    kv = rows + 100
    b = Batch([rows], [kv], group, 1, dim, 16, dtype, seed=dim)
    b.q[..., 3] = b.q[..., 3].abs() + 0.125
    for at in (20, kv - rows + rows // 2):
        b.k_pages[int(b.table[0, at // 16]), 0, at % 16, 3] = -math.inf
    out, lse = check(gpu_lib, b)
    assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()


# ---- more pieces than the partial results' workspace holds ----

def units_needed(rows, kv, group, kv_heads, dim, units):
    """What find_item (attention_plan.h) counts for a bf16 batch of the kernel with tiles of 128 rows: units of 16 rows of partial results."""
    tiles = [(-(-n * group // 128), 8, True) if n * group > 32 else (1, 1 if n * group <= 16 else 2, False) for n in rows]
    work = {m: sum(t * k for (t, _, many), k in zip(tiles, kv) if many == m) * kv_heads for m in (False, True)}

    def even(v, items, least):
        v = v / items
        return least if v <= least else (int(v) + 128) // 128 * 128

    piece = {False: even(work[False], 512, 128), True: even(work[False] + work[True], 2 * units, 512)}
    need = 0
    for (t, u, many), k in zip(tiles, kv):
        n = -(-k // piece[many])
        need += t * kv_heads * n * u if n > 1 else 0
    return need


@pytest.mark.parametrize("kv_heads", [8, 4, 1])
def test_more_pieces_than_the_workspace_holds(gpu_lib, kv_heads):
    """All of them are off then.  8 / kv_heads times as many sequences: up to 64, up to 256 and more are planned in ways of their own."""
    many, few = 62 * 8 // kv_heads, 8 // kv_heads
    rows, kv = [33] * many + [1] * few, [10000] * many + [16000] * few
    units = torch.cuda.get_device_properties(0).multi_processor_count
    assert units_needed(rows, kv, 1, kv_heads, 64, units) > 8192, units      # (sizes for 256 compute units)
    b = Batch(rows, [33] * many + [16000] + [1] * (few - 1), kv_heads, kv_heads, 64, 16, seed=kv_heads)
    b.table[:] = b.table[many].clone()        # the sequences share their pages
    b.kv = kv
    b.kv_lens = torch.tensor(kv, dtype=torch.int32, device=DEV)
    check(gpu_lib, b)
