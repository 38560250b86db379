"""Calls of the key/value cache whose time must not depend on what a neighbouring call's does not (timed as in test_gpu_pace.py)."""
import pytest
import torch

from test_gpu_pace import times

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# (measured, us, 4096 slots: sequences one by one 414, by halves 4.0, neighbours 2.9)
@pytest.mark.parametrize("S", [256, 4096, 65536])
def test_rows_of_slots_far_apart(gpu_lib, S):
    """Four rows of a wave in the first and the last of many slots, the ones between empty, beside four in the first two."""
    ctx = gpu_lib.KVContext(8, 2, 128, 16, torch.bfloat16, device=DEV)
    cache = torch.zeros(16, 2, 16, 128, dtype=torch.bfloat16, device=DEV)
    pages = ctx.pack_pages(cache, cache.clone())
    k = torch.randn(4, 2, 128, device=DEV).bfloat16()
    lens = torch.full((S,), 2, dtype=torch.int32, device=DEV)
    table = torch.zeros((S, 1), dtype=torch.int32, device=DEV)
    batches = []
    for second in (S - 1, 1):
        off = torch.zeros(S + 1, dtype=torch.int32)
        off[1:] = 2
        off[second + 1:] = 4
        table[second] = 1
        batches.append(ctx.pack_batch(off.to(DEV), lens, table))
    a, b = times(*[lambda batch=batch: ctx.moe_kv_append(k, k, pages, batch) for batch in batches])
    print(f"S = {S}: far {a:.2f} us, near {b:.2f} us")
    assert a <= 10 * b, (a, b)
