"""What a cache keeps: accumulated weights against 64 bits (bounds: keep_reference.weights), selection and compaction exactly."""
import math
import random

import pytest
import torch

import keep_reference as ref
from kv_reference import EPS, Batch, assert_within, attention, history

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def scores_of(b, seed=1):
    """Scores of a cache whose tokens have some; NaN where no token is."""
    g = torch.Generator().manual_seed(seed)
    n_pages = b.k_pages.shape[0]
    scores = torch.full((n_pages, b.kv_heads, b.page), math.nan)
    for s, kv in enumerate(b.kv):
        for i in range(min(-(-kv // b.page), b.table.shape[1])):
            if 0 <= (at := int(b.table[s, i])) < n_pages:
                n = min(b.page, kv - i * b.page)
                scores[at, :, :n] = torch.rand(b.kv_heads, n, generator=g)
    return scores.to(b.device)


def check_weights(lib, b, causal=True, window=0, decay=1.0, lse=None, scores=None):
    ctx, pages, batch = b.context(lib)
    if lse is None:
        lse = torch.empty(b.T, b.heads, device=DEV)
        ctx.moe_paged_attention(b.q, pages, batch, causal=causal, window=window, lse=lse)
    scores = scores_of(b) if scores is None else scores
    want, tol = ref.weights(b, lse, scores, causal, window, decay)
    got = ctx.moe_kv_weights(b.q, lse, pages, batch, scores.clone(), causal=causal, window=window, decay=decay)
    again = ctx.moe_kv_weights(b.q, lse, pages, batch, scores.clone(), causal=causal, window=window, decay=decay)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)                  # what no token has is left as it was
    assert_within(torch.where(nan, 0.0, got), torch.where(nan, 0.0, want), torch.where(nan, 0.0, tol), "scores")
    assert torch.equal(got.nan_to_num(-1.0), again.nan_to_num(-1.0))
    return got


@pytest.mark.parametrize("fmt", ["", "fp8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,page,kv_heads,group", [(16, 8, 1, 1), (32, 16, 2, 4), (64, 32, 2, 8), (80, 8, 1, 5), (96, 64, 3, 2), (112, 16, 1, 7),
                                                     (128, 16, 2, 8), (128, 128, 1, 16), (256, 8, 1, 4), (208, 32, 2, 3)])
def test_weights_types_and_layouts(gpu_lib, dim, page, kv_heads, group, dtype, fmt):
    b = Batch([1, 0, 4, 40, 1, 130], [1, 9, 4, 75, 300, 131], kv_heads * group, kv_heads, dim, page, dtype, fmt, seed=dim + group)
    check_weights(gpu_lib, b)
    check_weights(gpu_lib, b, window=50, decay=0.5)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 8, 33, 128, 2 ** 29])
@pytest.mark.parametrize("decay", [0.0, 1.0, 0.9])
@pytest.mark.parametrize("dtype,fmt,dim", [(torch.bfloat16, "", 64), (torch.bfloat16, "fp8", 128), (torch.float32, "", 64)])
def test_weights_masks(gpu_lib, causal, window, decay, dtype, fmt, dim):
    b = Batch([1, 3, 64, 20, 97, 300, 2], [5, 3, 64, 150, 230, 1000, 700], 8, 2, dim, 16, dtype, fmt, seed=window % 97)
    check_weights(gpu_lib, b, causal, window, decay)


@pytest.mark.parametrize("kv", [1, 2, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257, 1025, 20000])
@pytest.mark.parametrize("rows", [1, 2, 17])
def test_weights_at_every_length(gpu_lib, kv, rows):
    for dtype, fmt in ((torch.bfloat16, ""), (torch.bfloat16, "fp8"), (torch.float32, "")):
        if kv >= rows:
            check_weights(gpu_lib, Batch([rows], [kv], 8, 2, 128, 16, dtype, fmt, seed=kv))


@pytest.mark.parametrize("S", [64, 65, 256, 257, 700])
def test_weights_of_many_sequences(gpu_lib, S):
    r = random.Random(S)
    rows = [r.choice([0, 1, 1, 2, 5]) for _ in range(S)]
    kv = [r.choice([n, n + 1, n + 30, n + 150]) for n in rows]
    check_weights(gpu_lib, Batch(rows, kv, 4, 2, 64, 16, seed=S))


@pytest.mark.parametrize("dtype,fmt,dim", [(torch.bfloat16, "", 128), (torch.bfloat16, "fp8", 64), (torch.float32, "", 64), (torch.bfloat16, "", 256)])
def test_weights_of_a_draft_among_decode_rows(gpu_lib, dtype, fmt, dim):
    """More rows than the registers hold at once, in a batch that is one of few rows on average."""
    rows, kv = [1] * 40 + [20] + [1] * 23 + [3], [17 * i % 300 + 1 for i in range(40)] + [333] + [90] * 23 + [3]
    b = Batch(rows, kv, 8, 2, dim, 16, dtype, fmt, seed=dim)
    check_weights(gpu_lib, b)
    check_weights(gpu_lib, b, window=30, decay=0.5)
    check_weights(gpu_lib, b, causal=False, decay=0.0)


@pytest.mark.parametrize("dtype,fmt,dim", [(torch.bfloat16, "", 128), (torch.bfloat16, "fp8", 64), (torch.float32, "", 64), (torch.float32, "fp8", 256)])
@pytest.mark.parametrize("decode", [1, 17, 18, 60])
def test_weights_of_a_prompt_among_decode_rows(gpu_lib, decode, dtype, fmt, dim):
    """On both sides of where sequences of few rows have a launch of their own (here 17 and 18), a prompt, a piece of one and an empty sequence among them."""
    rows, kv = [1] * decode + [300, 0, 17], [29 * i % 400 + 1 for i in range(decode)] + [700, 5, 90]
    b = Batch(rows, kv, 8, 2, dim, 16, dtype, fmt, seed=decode)
    check_weights(gpu_lib, b)
    check_weights(gpu_lib, b, causal=False, window=100, decay=0.0)


def test_weights_where_nothing_is_seen(gpu_lib):
    """No tokens; fewer tokens than rows; pages given back; a table that ends early; rows whose lse is minus infinity."""
    b = Batch([2, 5, 1, 2, 3], [0, 2, 40, 100, 90], 4, 2, 64, 16, seed=11, dropped=((2, 0), (2, 1), (2, 2), (3, 5), (3, 6), (4, 2), (4, 3)))
    for causal in (True, False):
        check_weights(gpu_lib, b, causal=causal, window=20)
        check_weights(gpu_lib, b, causal=causal)
    b.table = b.table[:, :4].contiguous()
    check_weights(gpu_lib, b)
    b = Batch([3, 90], [40, 200], 4, 2, 64, 16, seed=12)
    lse = torch.randn(b.T, 4, device=DEV) + 4
    lse[1] = -math.inf
    lse[5:50, 2] = -math.inf
    check_weights(gpu_lib, b, lse=lse)
    lse[:] = -math.inf
    got = check_weights(gpu_lib, b, lse=lse, decay=0.0)
    assert (got[~torch.isnan(got)] == 0).all()


@pytest.mark.parametrize("last", [2 ** 31 - 1, 2 ** 31 - 255, 2 ** 31 - 256, 2 ** 30 + 77])
def test_weights_of_lengths_past_the_table(gpu_lib, last):
    """Positions come from the lengths as they are: rows far behind what the table reaches see all of that, or, with a window, nothing."""
    for dtype, fmt in ((torch.bfloat16, ""), (torch.float32, "fp8")):
        b = Batch([3, 40, 150], [300, 300, 300], 8, 2, 64, 16, dtype, fmt, seed=5)
        b.kv = [last, last, 5000]
        b.kv_lens.copy_(torch.tensor(b.kv, dtype=torch.int32))
        lse = torch.randn(b.T, 8, device=DEV) + 6
        scores = torch.rand(b.k_pages.shape[0], 2, 16, device=DEV)
        b.k_pages = torch.where(torch.isnan(b.k_pages.float()), torch.zeros_like(b.k_pages.float()), b.k_pages.float()).to(b.k_pages.dtype)
        if b.k_scales is not None:
            b.k_scales[b.k_scales == 255] = 127
        for causal, window, decay in ((True, 0, 1.0), (False, 0, 0.5), (True, 500, 0.5), (True, 2 ** 30, 0.0)):
            check_weights(gpu_lib, b, causal, window, decay, lse=lse, scores=scores)


def test_weights_of_a_token_are_its_own(gpu_lib):
    """A key that is not finite reaches its own sum alone, a row that is not finite those of the tokens that it sees, and with decay 0 no
    earlier score is read."""
    for dtype in (torch.bfloat16, torch.float32):
        for rows in (3, 50):
            b = Batch([rows], [rows + 100], 8, 1, 64, 16, dtype, seed=3)
            ctx, pages, batch = b.context(gpu_lib)
            lse = torch.randn(b.T, 8, device=DEV) + 5
            clean = ctx.moe_kv_weights(b.q, lse, pages, batch, torch.full_like(b.k_pages[..., 0], math.nan, dtype=torch.float32), decay=0.0)
            at = int(b.table[0, 70 // 16])
            was = b.k_pages[at, 0, 70 % 16].clone()
            b.k_pages[at, 0, 70 % 16, 3] = math.nan
            got = ctx.moe_kv_weights(b.q, lse, pages, batch, torch.full_like(clean, math.nan), decay=0.0)
            assert torch.isnan(got[at, 0, 70 % 16])
            got[at, 0, 70 % 16] = clean[at, 0, 70 % 16]
            assert torch.equal(got.nan_to_num(-1.0), clean.nan_to_num(-1.0))
            b.k_pages[at, 0, 70 % 16] = was
            b.q[rows - 2] = math.nan                     # the last row but one: all tokens but the last are NaN
            got = ctx.moe_kv_weights(b.q, lse, pages, batch, torch.full_like(clean, 5.0), decay=0.0)
            end = rows + 99
            place = int(b.table[0, end // 16]), 0, end % 16
            assert got[place] == clean[place]
            for j in (0, 50, end - 1):
                assert torch.isnan(got[int(b.table[0, j // 16]), 0, j % 16])


def lists(kv, page, hk, scores=None, seed=0, extra=3, dropped=()):
    g = torch.Generator().manual_seed(seed)
    need = [-(-k // page) for k in kv]
    n_pages = sum(need) + extra
    order = torch.randperm(n_pages, generator=g).tolist()
    table = torch.full((len(kv), max(need + [0]) + 1), -1, dtype=torch.int32)
    for s, n in enumerate(need):
        for i in range(n):
            at = order.pop()
            if (s, i) not in dropped:
                table[s, i] = at
    if scores is None:
        scores = torch.randn(n_pages, hk, page, generator=g)
    return scores.to(DEV), table.to(DEV), n_pages


def check_select(lib, kv, page, hk, budget, first=0, recent=0, make=None, **how):
    scores, table, n_pages = lists(kv, page, hk, **how)
    if make is not None:
        scores = make(scores)
    ctx = lib.KVContext(hk, hk, 32, page, torch.float32, device=DEV)
    batch = ctx.pack_batch(torch.zeros(len(kv) + 1, dtype=torch.int32, device=DEV), torch.tensor(kv, dtype=torch.int32, device=DEV), table)
    keep, lens = ctx.moe_kv_select(scores, batch, budget, first=first, recent=recent)
    want, want_lens = ref.select(scores, kv, table, page, n_pages, budget, first, recent)
    assert torch.equal(lens.cpu(), want_lens)
    assert torch.equal(keep.cpu(), want)
    return keep, lens


@pytest.mark.parametrize("page", [8, 16, 256])
@pytest.mark.parametrize("budget,first,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (7, 2, 3), (64, 4, 16), (100, 100, 0), (100, 0, 100), (999, 0, 0), (1024, 4, 64)])
def test_select(gpu_lib, page, budget, first, recent):
    kv = [0, 1, 6, 7, 8, 63, 64, 65, 500, 1023, 1024, 1025, 3000]
    check_select(gpu_lib, kv, page, 2, budget, first, recent)


@pytest.mark.parametrize("kv,budget", [([4096], 4095), ([4097], 1), ([20000], 300), ([20000, 5], 19999), ([70000], 5000), ([140000], 70000)])
def test_select_of_long_sequences(gpu_lib, kv, budget):
    check_select(gpu_lib, kv, 64, 2, budget, 1 if budget > 1 else 0, 0)


@pytest.mark.parametrize("kv", [[30000, 5, 16384, 16385, 0, 24577], [100000, 3000]])
@pytest.mark.parametrize("budget,first,recent", [(1, 0, 0), (2000, 4, 256), (16384, 0, 16000), (24576, 100, 100), (99999, 0, 0), (100000, 1, 1)])
def test_select_of_parts(gpu_lib, kv, budget, first, recent):
    """Sequences that several blocks share beside ones that a block has alone; holes, equal scores, two values."""
    check_select(gpu_lib, kv, 32, 1, budget, first, recent)
    check_select(gpu_lib, kv, 32, 2, budget, first, recent, dropped=[(0, i) for i in range(0, 900, 7)], seed=2)
    check_select(gpu_lib, kv, 32, 1, budget, first, recent, make=lambda x: torch.zeros_like(x))
    check_select(gpu_lib, kv, 32, 1, budget, first, recent, make=lambda x: (x > 1).float())


@pytest.mark.parametrize("values", [[0.0], [0.0, -0.0], [1.0, 0.0], [1.0, math.nan, -math.inf, -2.0], [math.inf, -math.inf, math.nan, 0.0, 3.5],
                                    [1e-45, 0.0, -1e-45, 1e-38], [1.0, 1.0 + 2.0 ** -23, 1.0 - 2.0 ** -24], [3.4e38, math.inf], [math.nan], [-math.inf, math.nan]])
def test_select_of_equal_and_strange_scores(gpu_lib, values):
    v = torch.tensor(values, device=DEV)

    def make(scores):
        g = torch.Generator().manual_seed(len(values))
        return v[torch.randint(len(values), scores.shape, generator=g).to(DEV)]

    for budget in (1, 5, 130, 700):
        check_select(gpu_lib, [200, 1500, 33], 16, 2, budget, min(2, budget - 1), 0, make=make)


def test_select_of_tokens_that_are_not_there(gpu_lib):
    kv = [100, 300, 50, 64]
    dropped = [(0, 0), (0, 6), (1, 3), (1, 4), (1, 18)] + [(2, i) for i in range(4)]
    for budget in (3, 40, 84, 85, 252, 260, 400):
        check_select(gpu_lib, kv, 16, 3, budget, 2, 1, dropped=dropped)
    scores, table, n_pages = lists(kv, 16, 2)
    table[3, 1], table[1, 2] = n_pages, 2 ** 31 - 1        # entries that name no page
    ctx = gpu_lib.KVContext(2, 2, 32, 16, torch.float32, device=DEV)
    lens = torch.tensor([100, 5000, -7, 64], dtype=torch.int32, device=DEV)      # past the table, negative
    batch = ctx.pack_batch(torch.zeros(5, dtype=torch.int32, device=DEV), lens, table)
    keep, kept = ctx.moe_kv_select(scores, batch, 30, first=3, recent=5)
    want, want_lens = ref.select(scores, lens.tolist(), table, 16, n_pages, 30, 3, 5)
    assert torch.equal(kept.cpu(), want_lens) and torch.equal(keep.cpu(), want)


def bits(t):
    """A tensor's bytes, so that NaN and codes compare as they are."""
    return t.contiguous().view(torch.uint8 if t.element_size() == 1 else torch.int16 if t.element_size() == 2 else torch.int32)


def check_compact(lib, b, keep, lens, first=None, scores=None):
    tensors = [t for t in (b.k_pages, b.v_pages, b.k_scales, b.v_scales, scores) if t is not None]
    want = ref.compact([bits(t).cpu() for t in tensors], b.kv, b.table, b.page, keep, lens, first)
    ctx, pages, batch = b.context(lib)
    ctx.moe_kv_compact(pages, batch, keep.to(DEV), lens.to(DEV), first=first.to(DEV) if first is not None else None, scores=scores)
    for got, ok in zip(tensors, want):
        assert torch.equal(bits(got).cpu(), ok)


def random_keep(kv, hk, budget, seed, start=None):
    r = random.Random(seed)
    keep, lens = torch.full((len(kv), hk, budget), -1, dtype=torch.int32), torch.zeros(len(kv), dtype=torch.int32)
    for s, n in enumerate(kv):
        lo = start[s] if start else 0
        lens[s] = m = min(budget, n - lo)
        for h in range(hk):
            keep[s, h, :m] = torch.tensor(sorted(r.sample(range(lo, n), m)), dtype=torch.int32)
    return keep, lens


@pytest.mark.parametrize("fmt", ["", "fp8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,page,hk", [(16, 8, 1), (32, 16, 2), (64, 32, 2), (80, 8, 1), (112, 16, 3), (128, 16, 2), (128, 256, 1), (208, 32, 2), (256, 8, 1)])
def test_compact_types_and_layouts(gpu_lib, dim, page, hk, dtype, fmt):
    kv = [1, 40, 0, 300, 129]
    for budget in (30, 128, 290):
        b = Batch([0] * 5, kv, hk, hk, dim, page, dtype, fmt, seed=dim)
        check_compact(gpu_lib, b, *random_keep(kv, hk, budget, budget), scores=scores_of(b) if budget != 128 else None)


@pytest.mark.parametrize("kv,budget", [([1000], 999), ([5000], 4900), ([5000], 2500), ([20000], 700), ([9000, 8000, 7000], 6999), ([700] * 40, 650)])
def test_compact_of_long_sequences(gpu_lib, kv, budget):
    """Nearly all, half and few of the tokens kept: what is written is read a little, or far, before; one hole at the front moves everything by one."""
    for fmt in ("", "fp8"):
        b = Batch([0] * len(kv), kv, 2, 2, 64, 16, torch.bfloat16, fmt, seed=budget)
        check_compact(gpu_lib, b, *random_keep(kv, 2, budget, 1), scores=scores_of(b))
    b = Batch([0] * len(kv), kv, 2, 2, 128, 16, seed=budget)
    keep = torch.stack([torch.arange(1, min(kv), dtype=torch.int32)] * len(kv))
    check_compact(gpu_lib, b, keep, torch.full((len(kv),), min(kv) - 1, dtype=torch.int32), scores=scores_of(b))


def test_compact_of_accepted_paths(gpu_lib):
    """The same rows for all heads, from a slot of each sequence's own; sequences that accept nothing, or everything; list ends past max_keep."""
    rows, kv = [16, 16, 16, 16, 3, 64], [16, 100, 513, 40, 3, 200]
    start = [k - n for k, n in zip(kv, rows)]
    b = Batch(rows, kv, 8, 4, 128, 16, seed=6)
    keep, lens = random_keep(kv, 1, 16, 3, start)
    keep = keep[:, 0].contiguous()
    keep[1], lens[1] = torch.arange(start[1], start[1] + 16), 16
    lens[2], lens[3] = 0, -5
    first = torch.tensor(start, dtype=torch.int32)
    want = lens.clamp(min=0)
    tensors = [b.k_pages, b.v_pages]
    ok = ref.compact([bits(t).cpu() for t in tensors], kv, b.table, 16, keep, want, first)
    ctx, pages, batch = b.context(gpu_lib)
    lens[0] = 1000                                    # (no more than max_keep count)
    ok[0], ok[1] = ref.compact([bits(t).cpu() for t in tensors], kv, b.table, 16, keep, torch.where(lens > 16, 16, want), first)
    ctx.moe_kv_compact(pages, batch, keep.to(DEV), lens.to(DEV), first=first.to(DEV))
    for got, o in zip(tensors, ok):
        assert torch.equal(bits(got).cpu(), o)


def test_compact_stays_within_the_sequences(gpu_lib):
    """Lists that are none (negative, past the sequence, past the table, descending): whatever they do, other sequences' pages stay."""
    kv = [64, 200, 300]
    b = Batch([0] * 3, kv, 2, 2, 64, 16, seed=8)
    g = torch.Generator().manual_seed(0)
    keep = torch.randint(-2 ** 31, 2 ** 31 - 1, (3, 2, 150), generator=g, dtype=torch.int32)
    keep[:, :, ::2] = torch.randint(0, 200, (3, 2, 75), generator=g, dtype=torch.int32)
    keep[1] = torch.arange(150)                           # nothing moves
    scores = scores_of(b)
    was = [bits(t).clone() for t in (b.k_pages, b.v_pages, scores)]
    ctx, pages, batch = b.context(gpu_lib)
    lens = torch.tensor([150, 150, 150], dtype=torch.int32, device=DEV)
    for first in (None, torch.tensor([0, 0, 2 ** 31 - 1], dtype=torch.int32, device=DEV), torch.tensor([-2 ** 31, 0, -9], dtype=torch.int32, device=DEV)):
        ctx.moe_kv_compact(pages, batch, keep.to(DEV), lens, first=first, scores=scores)
    mine = set(b.table[0].tolist() + b.table[2].tolist())
    others = [p for p in range(b.k_pages.shape[0]) if p not in mine]
    for t, w in zip((b.k_pages, b.v_pages, scores), was):
        assert torch.equal(bits(t)[others], w[others])


@pytest.mark.parametrize("dtype,fmt", [(torch.bfloat16, ""), (torch.bfloat16, "fp8"), (torch.float32, "")])
def test_evicted_cache_is_attended_to(gpu_lib, dtype, fmt):
    """Attention, its weights, the choice and the move, as a server runs them: then attention over what is left equals attention over the
    kept tokens of the old cache."""
    rows, kv, budget = [1, 40, 1, 200], [50, 300, 700, 200], 128
    b = Batch(rows, kv, 8, 2, 64, 16, dtype, fmt, seed=21)
    ctx, pages, batch = b.context(gpu_lib)
    lse = torch.empty(b.T, 8, device=DEV)
    ctx.moe_paged_attention(b.q, pages, batch, lse=lse)
    scores = ctx.moe_kv_weights(b.q, lse, pages, batch, torch.full((b.k_pages.shape[0], 2, 16), math.nan, device=DEV), decay=0.0)
    # a row's weights sum to one: the heads of a group give their number a row
    total = [sum(float(scores[int(b.table[s, j // 16]), h, j % 16]) for j in range(n)) for s, n in enumerate(kv) for h in range(2)]
    for s, n in enumerate(rows):
        for h in range(2):
            assert abs(total[2 * s + h] - 4 * n) < 1e-3 * n
    keep, lens = ctx.moe_kv_select(scores, batch, budget, first=4, recent=32)
    old = [t.clone() if t is not None else None for t in b.pages()]
    ctx.moe_kv_compact(pages, batch, keep, lens, scores=scores)
    assert lens.tolist() == [min(k, budget) for k in kv]
    # one more row a sequence, not appended: attention without a mask over what is left, against a gather of the kept tokens
    q = torch.randn(4, 8, 64, generator=torch.Generator().manual_seed(2)).to(dtype).to(DEV)
    after = ctx.pack_batch(torch.arange(5, dtype=torch.int32, device=DEV), lens, b.table)
    out = ctx.moe_paged_attention(q, pages, after, causal=False)
    for s, n in enumerate(kv):
        for h in range(2):
            tokens = keep[s, h, :int(lens[s])].long()
            k = history(old[0], old[2], b.table[s], n, h, 16)[0][tokens]
            v = history(old[1], old[3], b.table[s], n, h, 16)[0][tokens]
            w = torch.softmax(q[s, 4 * h:4 * h + 4].double() @ k.T / 8.0, 1)
            # a rounded result, rounded weights, and fp32 sums of the scores (64 + 8 half steps of sizes below 64) and outputs
            bound = EPS[dtype] * (w @ v).abs() + (EPS[torch.bfloat16] if dtype == torch.bfloat16 else 0.0) * (w @ v.abs()) + \
                (2 * 72 * 64 + 200) * 2.0 ** -24 * (w @ v.abs())
            assert ((out[s, 4 * h:4 * h + 4].double() - w @ v).abs() <= bound * 1.01).all()


def test_a_verified_draft_is_a_chain(gpu_lib):
    """Masks, attention to a tree, and the accepted path moved up: its rows' results are those of a causal chain of the same tokens."""
    parents, path = [-1, 0, 0, 1, 2, 2, 4, 6], [0, 2, 4, 6]
    n, past = len(parents), 77
    b = Batch([n], [past + n], 8, 2, 64, 16, seed=30)
    ctx, pages, batch = b.context(gpu_lib)
    ctx.moe_kv_append(b.k, b.v, pages, batch)
    masks, positions = ctx.moe_tree_masks(torch.tensor(parents, dtype=torch.int32, device=DEV), batch)
    assert [int(positions[i]) for i in path] == [past + i for i in range(4)]
    tree = ctx.moe_tree_attention(b.q, pages, batch, masks)
    keep = torch.tensor([[past + i for i in path]], dtype=torch.int32, device=DEV)
    lens, first = torch.tensor([4], dtype=torch.int32, device=DEV), torch.tensor([past], dtype=torch.int32, device=DEV)
    ctx.moe_kv_compact(pages, batch, keep, lens, first=first)
    chain = ctx.pack_batch(torch.tensor([0, 4], dtype=torch.int32, device=DEV), first + lens, b.table)
    out = ctx.moe_paged_attention(b.q[path].contiguous(), pages, chain)
    want, _, tol, _ = attention(b.q[path], b.pages(), [0, 4], [past + 4], b.table, 16)
    assert_within(out, want, tol)
    assert_within(tree[path], want, tol)
    # and the cache holds what appending the chain would have left
    k, v = ctx.moe_kv_gather(pages, chain, T=4)
    assert torch.equal(k, b.k[path]) and torch.equal(v, b.v[path])


@pytest.mark.parametrize("dtype,group", [(torch.bfloat16, 8), (torch.bfloat16, 5), (torch.float32, 4)])
def test_weights_of_rows_at_the_edges_of_stages(gpu_lib, dtype, group):
    """Rows that are kept in registers, those that LDS holds, and more; one to three stages of them, whole and with a rest."""
    edges = [1, 2, 3, 4, 12, 13, 16, 17, 24, 25, 26, 31, 32, 33, 51, 52, 63, 64, 65, 96, 97, 103]
    check_weights(gpu_lib, Batch(edges, [n + 37 * i % 500 for i, n in enumerate(edges)], 2 * group, 2, 64, 16, dtype, seed=group))
    check_weights(gpu_lib, Batch([33, 64, 96], [3000, 64, 2000], group, 1, 128, 64, dtype, "fp8", seed=group), window=200, decay=0.25)


def test_weights_of_long_prompts(gpu_lib):
    """Tiles that many stretches share, behind a prompt's start and a history; beside decode and held rows."""
    for dtype, fmt, dim in ((torch.bfloat16, "", 128), (torch.bfloat16, "fp8", 64), (torch.float32, "", 64)):
        rows, kv = [1500, 1, 20, 700], [1500, 2000, 900, 3100]
        b = Batch(rows, kv, 8, 2, dim, 16, dtype, fmt, seed=dim)
        check_weights(gpu_lib, b)
        check_weights(gpu_lib, b, window=333, decay=0.5)
        check_weights(gpu_lib, b, causal=False, decay=0.0)


def test_weights_of_more_sequences_than_have_slots(gpu_lib):
    """Prompts in the first and the last of 2400 sequences: the last ones' tiles have no slots for partial sums and are not shared."""
    S = 2400
    rows = [1] * S
    for s in (0, 1, 255, 256, 1000, 2047, 2048, 2300, S - 1):
        rows[s] = 150
    kv = [n + (200 if n > 1 else s % 7) for s, n in enumerate(rows)]
    check_weights(gpu_lib, Batch(rows, kv, 4, 1, 16, 16, seed=1))


def graphed(f):
    """f captured: a function that replays it.  Its first call runs in the graph, so what a context clears belongs to it."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        f()
    return g.replay


@pytest.mark.parametrize("warm", [False, True])
def test_captured_calls_replay(gpu_lib, warm):
    """A pass of all calls in a graph, replayed over new descriptors with eager calls of the same context and waits between."""
    b = Batch([30, 300, 1, 8], [200, 900, 500, 70], 8, 2, 64, 16, seed=40)
    ctx, pages, batch = b.context(gpu_lib)
    parents = torch.tensor([i - 1 if n > 64 else (i - 1) // 2 for n in b.rows for i in range(n)], dtype=torch.int32, device=DEV)
    lse, out = torch.empty(b.T, 8, device=DEV), torch.empty(b.T, 8, 64, dtype=torch.bfloat16, device=DEV)
    scores = scores_of(b)
    masks, positions = torch.empty(b.T, 1, dtype=torch.int64, device=DEV), torch.empty(b.T, dtype=torch.int32, device=DEV)
    keep, lens = torch.empty(4, 2, 150, dtype=torch.int32, device=DEV), torch.empty(4, dtype=torch.int32, device=DEV)
    start = [t.clone() for t in (b.k_pages, b.v_pages, scores)]

    def calls():
        ctx.moe_tree_masks(parents, batch, masks=masks, positions=positions)
        ctx.moe_tree_attention(b.q, pages, batch, masks, out=out)
        ctx.moe_paged_attention(b.q, pages, batch, lse=lse)
        ctx.moe_kv_weights(b.q, lse, pages, batch, scores)
        ctx.moe_kv_select(scores, batch, 150, first=2, recent=70, keep=keep, keep_lens=lens)
        ctx.moe_kv_compact(pages, batch, keep, lens, scores=scores)

    def reset():
        for t, w in zip((b.k_pages, b.v_pages, scores), start):
            t.copy_(w)

    def results():
        return [bits(t).clone() for t in (masks, positions, out, scores, keep, lens, b.k_pages, b.v_pages)]

    if warm:
        calls()
        torch.cuda.synchronize()
    replay = graphed(calls)
    for i, kv in enumerate(([200, 900, 500, 70], [31, 300, 2, 9], [180, 880, 512, 64], [200, 900, 500, 70])):
        b.kv_lens.copy_(torch.tensor(kv, dtype=torch.int32))
        reset()
        replay()
        got = results()
        reset()
        calls()
        for x, y in zip(got, results()):
            assert torch.equal(x, y), i
        torch.cuda.synchronize()


def test_calls_on_another_stream(gpu_lib):
    """A context's calls follow the current stream."""
    b = Batch([40, 1, 200], [300, 700, 200], 8, 2, 64, 16, seed=41)
    ctx, pages, batch = b.context(gpu_lib)
    lse = torch.empty(b.T, 8, device=DEV)
    ctx.moe_paged_attention(b.q, pages, batch, lse=lse)
    want = ctx.moe_kv_weights(b.q, lse, pages, batch, scores_of(b))
    keep, lens = ctx.moe_kv_select(want, batch, 100, recent=10)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        scores = scores_of(b)
        for _ in range(3):
            late = torch.randn(2048, 2048, device=DEV) @ torch.randn(2048, 2048, device=DEV)
        scores += 0.0 * late[0, 0].nan_to_num()
        got = ctx.moe_kv_weights(b.q, lse, pages, batch, scores)
        keep2, lens2 = ctx.moe_kv_select(got, batch, 100, recent=10)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got.nan_to_num(-1.0), want.nan_to_num(-1.0)) and torch.equal(keep, keep2) and torch.equal(lens, lens2)
