"""The weights that verified drafts give to a cache: after the accepted paths have moved up, their rows are chains."""
import copy
import math
import random

import pytest
import torch

import keep_reference as ref
from kv_reference import Batch, assert_within
from test_gpu_keep import scores_of
from test_gpu_tree import parents_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype,fmt,group", [(torch.bfloat16, "", 8), (torch.bfloat16, "fp8", 4), (torch.float32, "", 2)])
@pytest.mark.parametrize("window,decay", [(0, 1.0), (0, 0.0), (5, 0.5), (40, 1.0)])
def test_weights_of_accepted_rows(gpu_lib, dtype, fmt, group, window, decay):
    """Trees, their attention, the accepted paths moved up with their scores, and the weights of the accepted rows with the lse that the trees' attention
    gave them: scores by the definition over the chains, whose rows give one to each of a group's heads."""
    rows, past = [16, 30, 1, 64, 8], [70, 0, 33, 500, 3]
    b = Batch(rows, [p + n for p, n in zip(past, rows)], 2 * group, 2, 64, 16, dtype, fmt, seed=group)
    ctx, pages, batch = b.context(gpu_lib)
    parents = parents_of(rows, "tree", 4)
    masks, positions = ctx.moe_tree_masks(torch.tensor(parents, dtype=torch.int32, device=DEV), batch, window=window)
    lse = torch.empty(b.T, b.heads, device=DEV)
    ctx.moe_tree_attention(b.q, pages, batch, masks, positions=positions, window=window, lse=lse)
    # a path of each tree, as far as it is accepted; the last tree's draft is refused whole
    r = random.Random(7)
    paths = [ref.paths(parents[o:o + n])[r.randrange(n // 2, n)] for o, n in zip(b.offsets, rows)]
    paths[-1] = []
    keep = torch.full((len(rows), max(map(len, paths))), -1, dtype=torch.int32)
    for s, path in enumerate(paths):
        keep[s, :len(path)] = torch.tensor(path, dtype=torch.int32) + past[s]
    lens, first = torch.tensor([len(p) for p in paths], dtype=torch.int32, device=DEV), torch.tensor(past, dtype=torch.int32, device=DEV)
    scores = scores_of(b)
    ctx.moe_kv_compact(pages, batch, keep.to(DEV), lens, first=first, scores=scores)
    taken = [o + i for o, path in zip(b.offsets, paths) for i in path]
    chain = copy.copy(b)
    chain.rows, chain.q, chain.T = [len(p) for p in paths], b.q[taken].contiguous(), len(taken)
    chain.kv = [p + n for p, n in zip(past, chain.rows)]
    chain.offsets = [sum(chain.rows[:s]) for s in range(len(rows) + 1)]
    chain.kv_lens, chain.row_offsets = first + lens, torch.tensor(chain.offsets, dtype=torch.int32, device=DEV)
    after = ctx.pack_batch(chain.row_offsets, chain.kv_lens, b.table)
    want, tol = ref.weights(chain, lse[taken], scores, True, window, decay)
    got = ctx.moe_kv_weights(chain.q, lse[taken].contiguous(), pages, after, scores.clone(), window=window, decay=decay)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    assert_within(torch.where(nan, 0.0, got), torch.where(nan, 0.0, want), torch.where(nan, 0.0, tol), "scores")
    if decay == 0.0:
        # every row's weights sum to one, by the bound of its lse and of a weight: 2^-10 is far above both in 32 bits, a token too many or too few far above that
        for s, kv in enumerate(chain.kv):
            for h in range(2 if chain.rows[s] else 0):
                total = math.fsum(float(got[int(b.table[s, j // 16]), h, j % 16]) for j in range(kv))
                assert abs(total - group * chain.rows[s]) <= 2.0 ** -10 * group * chain.rows[s]
