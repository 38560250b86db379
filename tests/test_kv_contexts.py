"""What the key/value cache's contexts refuse beside what test_kv_abi.py has (no GPU)."""
import pytest
import torch

from paper_2510_08055_amd import binding
from test_kv_abi import SHAPE, Call


def cache(ctx, n=3):
    shape = (n, ctx.kv_heads, ctx.page, ctx.dim)
    pages = [torch.zeros(shape).to(ctx.page_dtype) for _ in range(2)]
    scales = [torch.zeros(shape[:3], dtype=torch.uint8) for _ in range(2)] if ctx.fp8 else []
    off, lens, table = (torch.zeros(s, dtype=torch.int32) for s in ((3,), (2,), (2, 4)))
    return ctx.pack_pages(*pages, *scales), ctx.pack_batch(off, lens, table)


def calls(ctx, pages, batch, T=3):
    q, k = torch.zeros(T, ctx.heads, ctx.dim, dtype=ctx.dtype), torch.zeros(T, ctx.kv_heads, ctx.dim, dtype=ctx.dtype)
    return [lambda: ctx.moe_kv_append(k, k, pages, batch), lambda: ctx.moe_kv_gather(pages, batch, T=T),
            lambda: ctx.moe_kv_gather(pages, batch, k=k, v=k.clone()), lambda: ctx.moe_paged_attention(q, pages, batch)]


def make(heads=4, kv_heads=2, dim=32, page=8, dtype=torch.float32, fmt=""):
    return binding.KVContext(heads, kv_heads, dim, page, dtype, kv_format=fmt, device="cpu")


@pytest.mark.parametrize("other", [{"kv_heads": 4}, {"dim": 64}, {"page": 16}, {"dtype": torch.bfloat16}, {"fmt": "fp8"}])
def test_pages_of_another_layout_are_refused(other):
    """The struct holds pointers: a context of another layout would read and write past the tensors."""
    a, b = make(), make(**other)
    for mine, theirs in ((a, b), (b, a)):
        pages, _ = cache(theirs)
        _, batch = cache(mine)
        for f in calls(mine, pages, batch):
            with pytest.raises(ValueError, match="pages packed for"):
                f()


def test_structs_that_were_not_packed_are_refused():
    ctx = make()
    pages, batch = cache(ctx)
    for bad in (None, binding.CKVPages(pages.k_pages, pages.v_pages, None, None, 3), binding.KVPages()):
        for f in calls(ctx, bad, batch):
            with pytest.raises(ValueError, match="pages packed for"):
                f()
    for bad in (None, binding.CKVBatch(), binding.KVBatch()):
        for f in calls(ctx, pages, bad):
            with pytest.raises(ValueError, match="a batch packed on"):
                f()


def test_contexts_of_the_same_layout_share_pages():
    """Such a call gets as far as the GPU that is not there; query heads may differ, and so may the dtype beside FP8 pages."""
    for a, b in ((make(), make(heads=8)), (make(fmt="fp8"), make(dtype=torch.bfloat16, fmt="fp8"))):
        pages, batch = cache(a)
        for f in calls(b, pages, batch):
            with pytest.raises(ValueError, match="the kernels run on a GPU"):
                f()


def test_sizes_past_32_bits_are_refused():
    """Their lower bits alone would be legal sizes: a window of 2^32 + 5 would be one of 5."""
    ctx = make()
    pages, batch = cache(ctx)
    q = torch.zeros(3, 4, 32)
    for window in (2 ** 32 + 5, 2 ** 32, 2 ** 31, -2 ** 32 + 1):
        with pytest.raises(ValueError, match="does not fit 32 bits"):
            ctx.moe_paged_attention(q, pages, batch, window=window)
    for name, v in (("heads", 4), ("kv_heads", 2), ("dim", 32), ("page", 8)):
        with pytest.raises(ValueError, match="does not fit 32 bits"):
            make(**{name: 2 ** 32 + v})
    with pytest.raises(ValueError, match="does not fit 32 bits"):
        binding.kv_workspace_bytes(2 ** 32 + 4, 2, 32, 8, torch.float32)


def test_calls_of_more_blocks_than_a_launch_has_are_refused():
    """Legal in every other number: 2^30 rows of one head, and 2^22 - 1 sequences of a row of 256 heads."""
    c = Call(heads=1, kv_heads=1, dim=16)
    batch = {"n_seqs": 2 ** 22 - 1}
    assert c.status("append", T=2 ** 30) == SHAPE and c.status("gather", T=2 ** 30) == SHAPE
    assert c.status("append", T=2 ** 30, batch=batch) == SHAPE
    for fmt, dtype in ((0, 1), (1, 1), (0, 0), (1, 0)):
        c = Call(heads=256, kv_heads=256, dim=32, fmt=fmt, dtype=dtype)
        for what in ("append", "gather", "attention"):
            assert c.status(what, T=2 ** 22, batch=batch) == SHAPE, (what, fmt, dtype)
