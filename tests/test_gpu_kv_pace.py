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


# A prompt's chunk beside decode rows takes no longer than either alone, one after the other, however many the decode rows, the heads of a group
# or the slots without rows (measured, us, together / the two alone: 16-row tiles for all 479 / 222, 443 / 215 and 322 / 105, tiles of 128 for the
# chunk 199, 197 and 94)
@pytest.mark.parametrize("kv_heads,decode,empty", [(32, 64, 0), (8, 256, 0), (8, 32, 223)])
def test_a_chunk_among_decode_rows(gpu_lib, kv_heads, decode, empty):
    heads, dim, page, P, past = 32, 128, 16, 512, 7680
    ctx = gpu_lib.KVContext(heads, kv_heads, dim, page, torch.bfloat16, device=DEV)
    lens = [512 + i * 37 % 512 for i in range(decode)] + [past + P] + [0] * empty
    need = [-(-n // page) for n in lens]
    k, v = (torch.randn(sum(need), kv_heads, page, dim, device=DEV).bfloat16() for _ in range(2))
    pages = ctx.pack_pages(k, v)
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
    for s, n in enumerate(need):
        table[s, :n] = torch.arange(n) + sum(need[:s])

    def call(rows, which):
        off = torch.tensor([0] + rows).cumsum(0).int().to(DEV)
        batch = ctx.pack_batch(off, torch.tensor([lens[s] for s in which], dtype=torch.int32, device=DEV), table[which].to(DEV))
        q = torch.randn(sum(rows), heads, dim, device=DEV).bfloat16()
        out = torch.empty_like(q)
        return lambda: ctx.moe_paged_attention(q, pages, batch, out=out)

    every = list(range(len(lens)))
    both, chunk, rest = times(call([1] * decode + [P] + [0] * empty, every), call([P], [decode]), call([1] * decode, every[:decode]))
    print(f"together {both:.1f} us, chunk {chunk:.1f} us, decode rows {rest:.1f} us")
    assert both <= 1.4 * (chunk + rest), (both, chunk, rest)
