"""What a cache keeps, on the ways that only large calls take: many long sequences, lists of more words than the counters have."""
import pytest
import torch

import keep_reference as ref
from kv_reference import Batch
from test_gpu_keep import bits, graphed, lists, random_keep, scores_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def units():
    return torch.cuda.get_device_properties(DEV).multi_processor_count


def check_select(lib, scores, kv, table, page, budget, first, recent):
    hk = scores.shape[1]
    ctx = lib.KVContext(hk, hk, 32, page, torch.float32, device=DEV)
    batch = ctx.pack_batch(torch.zeros(len(kv) + 1, dtype=torch.int32, device=DEV), torch.tensor(kv, dtype=torch.int32, device=DEV), table)
    keep, lens = ctx.moe_kv_select(scores, batch, budget, first=first, recent=recent)
    want, want_lens = ref.select(scores, kv, table, page, scores.shape[0], budget, first, recent)
    assert torch.equal(lens.cpu(), want_lens)
    assert torch.equal(keep.cpu(), want)


@pytest.mark.parametrize("budget,first,recent", [(1, 0, 0), (4096, 4, 256), (16385, 0, 16000), (40000, 100, 100), (49153, 1, 0)])
@pytest.mark.parametrize("scores", ["random", "holes", "equal", "two values"])
def test_select_of_many_long_sequences(gpu_lib, scores, budget, first, recent):
    """As many sequences and heads as there are units: a block has each to itself, in registers up to 49152 tokens, longer ones count by count."""
    hk, page = 8, 32
    kv = [16384, 16385, 20000, 32767, 45057, 49151, 49152, 49153, 65537, 70001]
    kv += [s % 40 for s in range(-(-units() // hk) - len(kv))]
    assert len(kv) * hk >= units()
    dropped = {(s, i) for s in range(10) for i in range(s, 3000, 7)} if scores == "holes" else ()
    x, table, _ = lists(kv, page, hk, dropped=dropped, seed=budget)
    if scores == "equal":
        x = torch.full_like(x, -0.5)
    elif scores == "two values":
        x = (x > 0.5).float()
    check_select(gpu_lib, x, kv, table, page, budget, first, recent)


@pytest.mark.parametrize("budget,first,recent", [(1, 0, 0), (5000, 4, 256), (60000, 0, 0)])
def test_select_of_tables_that_the_workspace_does_not_hold(gpu_lib, budget, first, recent):
    """Few sequences in parts need words for every token that a table could name; where there are too few, a block has each sequence to itself."""
    page, hk = 256, 2
    kv = [70000, 5, 16385, 49152, 0]
    x, table, _ = lists(kv, page, hk, seed=budget, dropped=[(0, 3), (0, 200), (2, 0)])
    wide = torch.full((len(kv), 2 ** 20 // page), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    assert len(kv) * hk < units() and len(kv) * hk * 2 ** 20 * 4 > gpu_lib.kv_workspace_bytes(hk, hk, 32, page, torch.float32)
    check_select(gpu_lib, x, kv, wide, page, budget, first, recent)
    kv[4] = 2 ** 20 + 77                                  # past the table; of all that only its last page is there
    wide[4, -1] = int((~torch.isin(torch.arange(x.shape[0], device=DEV), wide.long())).nonzero()[0])
    check_select(gpu_lib, x, kv, wide, page, budget, first, recent)



def words(max_keep, items, dim, dtype):
    """Tiles of a list, and the words that all of them take (a word to a tile and two counters; 65536 are there)."""
    lanes = next(n for n in (4, 8, 16, 32, 64) if n >= dim * torch.empty(0, dtype=dtype).element_size() // 16)
    tiles = -(-max_keep // (256 // lanes * 8))
    return tiles, items * (tiles + 2)


def moved(b, keep, lens, scores):
    """What a compaction leaves, as bytes."""
    return ref.compact([bits(t).cpu() for t in (b.k_pages, b.v_pages, scores)], b.kv, b.table, b.page, keep, lens, None)


def assert_moved(b, scores, want):
    for got, ok in zip((b.k_pages, b.v_pages, scores), want):
        assert torch.equal(bits(got).cpu(), ok)


LAYOUTS = [([1000, 700, 900], 600, True), ([400] * 7, 300, False), ([5000], 4900, True), ([0, 3, 1500], 1400, True), ([1000, 700, 900], 600, True),
           ([260] * 40, 257, True), ([3000, 2000], 129, False), ([5000], 4900, True)]


def layout(kv, budget, per_head, seed):
    b = Batch([0] * len(kv), kv, 2, 2, 128, 16, seed=seed)
    keep, lens = random_keep(kv, 2, budget, seed)
    if not per_head:
        keep = keep[:, 0].contiguous()
    tiles, n = words(budget, 2 * len(kv), 128, torch.bfloat16)
    assert tiles > 1 and n <= 65536
    return b, keep, lens, scores_of(b)


def test_compact_again_and_again(gpu_lib):
    """Lists of several tiles by one context, in layouts that put counters where others had marks: every call finds what the one before left."""
    made = [layout(*how, seed=i) for i, how in enumerate(LAYOUTS)]
    want = [moved(*x) for x in made]
    ctx = made[0][0].context(gpu_lib)[0]
    for b, keep, lens, scores in made:
        ctx.moe_kv_compact(ctx.pack_pages(*b.pages()), ctx.pack_batch(b.row_offsets, b.kv_lens, b.table), keep.to(DEV), lens.to(DEV), scores=scores)
    for (b, _, _, scores), w in zip(made, want):
        assert_moved(b, scores, w)


@pytest.mark.parametrize("warm", [False, True])
def test_captured_compaction_of_tiles_replays(gpu_lib, warm):
    """A graph of lists of several tiles, replayed over new lists, with eager calls of other layouts between."""
    b, keep, lens, scores = layout([1000, 700, 900], 600, True, 3)
    other, other_keep, other_lens, other_scores = layout([400] * 7, 300, False, 4)
    ctx, pages, batch = b.context(gpu_lib)
    lists_of, lens_of = torch.empty_like(keep, device=DEV), torch.empty_like(lens, device=DEV)
    start = [t.clone() for t in (b.k_pages, b.v_pages, scores, other.k_pages, other.v_pages, other_scores)]
    held = (b.k_pages, b.v_pages, scores, other.k_pages, other.v_pages, other_scores)

    def eager():
        ctx.moe_kv_compact(ctx.pack_pages(*other.pages()), ctx.pack_batch(other.row_offsets, other.kv_lens, other.table), other_keep.to(DEV),
                           other_lens.to(DEV), scores=other_scores)

    other_want = moved(other, other_keep, other_lens, other_scores)
    if warm:
        eager()
        torch.cuda.synchronize()
    replay = graphed(lambda: ctx.moe_kv_compact(pages, batch, lists_of, lens_of, scores=scores))
    for i in range(4):
        for t, w in zip(held, start):
            t.copy_(w)
        keep, lens = random_keep(b.kv, 2, 600, 50 + i)
        lists_of.copy_(keep)
        lens_of.copy_(lens)
        want = moved(b, keep, lens, scores)
        replay()
        if i % 2:
            eager()
            assert_moved(other, other_scores, other_want)
        assert_moved(b, scores, want)


@pytest.mark.parametrize("dim,dtype,budget,seqs", [(128, torch.bfloat16, 1000, 1700), (256, torch.float32, 200, 1850), (16, torch.bfloat16, 2000, 2750)])
def test_compact_of_more_lists_than_there_are_words(gpu_lib, dim, dtype, budget, seqs):
    """Lists whose tiles outnumber the counters: a block takes a sequence and head, tile after tile.  Then by the same context few that do not."""
    hk = 4
    tiles, n = words(budget, seqs * hk, dim, dtype)
    assert tiles > 3 and n > 65536
    long = {0: 3 * budget, 7: budget + 1, 700: budget, seqs - 1: budget + budget // 2}
    kv = [long.get(s, s % 5) for s in range(seqs)]
    b = Batch([0] * seqs, kv, hk, hk, dim, 16, dtype, seed=dim)
    keep, lens = random_keep(kv, hk, budget, 2)
    scores = scores_of(b)
    want = moved(b, keep, lens, scores)
    ctx, pages, batch = b.context(gpu_lib)
    ctx.moe_kv_compact(pages, batch, keep.to(DEV), lens.to(DEV), scores=scores)
    assert_moved(b, scores, want)
    few = Batch([0], [3 * budget], hk, hk, dim, 16, dtype, seed=1)
    keep, lens = random_keep(few.kv, hk, budget, 3)
    scores = scores_of(few)
    want = moved(few, keep, lens, scores)
    ctx.moe_kv_compact(ctx.pack_pages(*few.pages()), ctx.pack_batch(few.row_offsets, few.kv_lens, few.table), keep.to(DEV), lens.to(DEV), scores=scores)
    assert_moved(few, scores, want)
