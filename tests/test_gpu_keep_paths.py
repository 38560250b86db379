"""What a cache keeps, on the ways that only large calls take: many long sequences, lists of more words than the counters have."""
import pytest
import torch

import keep_reference as ref
from test_gpu_keep import lists

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

