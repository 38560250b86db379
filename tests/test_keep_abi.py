"""Host-side checks of the tree, weight and keep entry points (no GPU): bad arguments are refused before any launch."""
import math

import pytest
import torch

from paper_2510_08055_amd import binding
from test_kv_abi import ALIGN, FAKE, NULL, SHAPE
from test_kv_abi import Call as KVCall
from test_kv_contexts import cache, make


class Call(KVCall):
    def keep_status(self, what, T=4, pages=None, batch=None, ctx=True, q=FAKE, ldq=None, opt=(1, 0), lse=FAKE, scores=FAKE, words=1,
                    masks=FAKE, positions=FAKE, parents=FAKE, decay=1.0, n_pages=10, select=(8, 1, 2), keep=FAKE, lens=FAKE, first=None,
                    max_keep=8, per_head=1, tree=True, options=True):
        p, b = binding.CKVPages(FAKE, FAKE, FAKE, FAKE, 10), binding.CKVBatch(FAKE, FAKE, FAKE, 2, 8)
        for struct, change in ((p, pages), (b, batch)):
            for k, v in (change or {}).items():
                setattr(struct, k, v)
        c = self.ctx if ctx else None
        ldq = self.cfg.heads * self.cfg.dim if ldq is None else ldq
        if what == "masks":
            return self.lib.moe_tree_masks(c, parents, T, b, words, opt[1], masks, positions, None)
        if what == "tree":
            return self.lib.moe_tree_attention(c, q, ldq, T, p, b, binding.CTree(masks, positions, words) if tree else None,
                                               binding.CAttentionOptions(opt[0], opt[1], None) if options else None, FAKE, ldq, None, None)
        if what == "weights":
            return self.lib.moe_kv_weights(c, q, ldq, lse, T, p, b, binding.CWeightsOptions(opt[0], opt[1], decay) if options else None, scores, None)
        if what == "select":
            return self.lib.moe_kv_select(c, scores, n_pages, b, binding.CSelectOptions(*select) if options else None, keep, lens, None)
        return self.lib.moe_kv_compact(c, p, b, binding.CKVKeep(keep, lens, first, max_keep, per_head) if options else None, scores, None)


@pytest.mark.parametrize("what", ["masks", "tree", "weights"])
def test_calls_with_rows(what):
    c = Call(fmt=1)
    assert c.keep_status(what, T=0) == 0
    assert c.keep_status(what, T=0, batch={"row_offsets": None, "n_seqs": 0, "max_pages": 0}) == 0
    assert c.keep_status(what, ctx=False) == NULL
    assert c.keep_status(what, T=-1) == SHAPE and c.keep_status(what, T=2 ** 31) == SHAPE and c.keep_status(what, T=2 ** 40) == SHAPE
    assert c.keep_status(what, opt=(1, -1)) == SHAPE and c.keep_status(what, opt=(1, 2 ** 31 - 1)) == SHAPE
    for field in ("row_offsets", "kv_lens"):
        assert c.keep_status(what, batch={field: None}) == NULL and c.keep_status(what, batch={field: FAKE + 2}) == ALIGN
    assert c.keep_status(what, batch={"n_seqs": 0}) == SHAPE and c.keep_status(what, batch={"n_seqs": -1}) == SHAPE
    assert c.keep_status(what, batch={"n_seqs": 2 ** 31}) == SHAPE
    if what != "masks":
        assert c.keep_status(what, options=False) == NULL
        assert c.keep_status(what, q=None) == NULL and c.keep_status(what, q=FAKE + 8) == ALIGN
        assert c.keep_status(what, ldq=500) == SHAPE and c.keep_status(what, ldq=516) == ALIGN
        for field in ("k_pages", "v_pages", "k_scales", "v_scales"):
            assert c.keep_status(what, pages={field: None}) == NULL and c.keep_status(what, pages={field: FAKE + 8}) == ALIGN
        assert c.keep_status(what, batch={"page_table": None}) == NULL and c.keep_status(what, batch={"max_pages": 2 ** 31}) == SHAPE
    if what != "weights":
        for words in (0, -1, 17):
            assert c.keep_status(what, words=words) == SHAPE, words
        assert c.keep_status(what, masks=None) == NULL and c.keep_status(what, masks=FAKE + 4) == ALIGN
        assert c.keep_status(what, positions=FAKE + 2, opt=(1, 5)) == ALIGN


def test_trees():
    c = Call()
    assert c.keep_status("masks", parents=None) == NULL and c.keep_status("masks", parents=FAKE + 1) == ALIGN
    assert c.keep_status("tree", tree=False) == NULL
    assert c.keep_status("tree", opt=(0, 0)) == SHAPE and c.keep_status("tree", opt=(2, 0)) == SHAPE
    assert c.keep_status("tree", opt=(1, 4), positions=None) == NULL


def test_weights():
    c = Call()
    assert c.keep_status("weights", opt=(2, 0)) == SHAPE
    for decay in (-0.5, 1.5, math.nan, math.inf):
        assert c.keep_status("weights", decay=decay) == SHAPE
    assert c.keep_status("weights", lse=None) == NULL and c.keep_status("weights", lse=FAKE + 2) == ALIGN
    assert c.keep_status("weights", ldq=2 ** 23 + 8) == SHAPE
    assert c.keep_status("weights", scores=None) == NULL and c.keep_status("weights", scores=FAKE + 8) == ALIGN


@pytest.mark.parametrize("what", ["select", "compact"])
def test_calls_without_rows(what):
    c = Call(fmt=1)
    assert c.keep_status(what, ctx=False) == NULL and c.keep_status(what, options=False) == NULL
    assert c.keep_status(what, batch={"row_offsets": None, "n_seqs": 0}) == 0      # no sequences: a no-op
    for field in ("kv_lens", "page_table"):
        assert c.keep_status(what, batch={field: None}) == NULL and c.keep_status(what, batch={field: FAKE + 2}) == ALIGN
    assert c.keep_status(what, batch={"n_seqs": -1}) == SHAPE and c.keep_status(what, batch={"n_seqs": 2 ** 31}) == SHAPE
    assert c.keep_status(what, batch={"max_pages": -1}) == SHAPE and c.keep_status(what, batch={"max_pages": 2 ** 31}) == SHAPE
    assert c.keep_status(what, scores=FAKE + 8) == ALIGN
    assert c.keep_status(what, keep=None) == NULL and c.keep_status(what, lens=None) == NULL
    assert c.keep_status(what, keep=FAKE + 2) == ALIGN and c.keep_status(what, lens=FAKE + 2) == ALIGN


def test_select():
    c = Call()
    assert c.keep_status("select", scores=None) == NULL
    for n in (0, -1, 2 ** 31):
        assert c.keep_status("select", n_pages=n) == SHAPE
    for bad in ((0, 0, 0), (-4, 0, 0), (8, -1, 0), (8, 0, -1), (8, 5, 4), (2 ** 31 - 1, 0, 0), (8, 2 ** 31 - 1, 2 ** 31 - 1)):
        assert c.keep_status("select", select=bad) == SHAPE, bad
    many = Call(heads=4096, kv_heads=4096, dim=16)
    assert many.keep_status("select", batch={"n_seqs": 2 ** 20, "max_pages": 1}) == SHAPE      # more blocks than a launch has


def test_compact():
    c = Call(fmt=1)
    for field in ("k_pages", "v_pages", "k_scales", "v_scales"):
        assert c.keep_status("compact", pages={field: None}) == NULL and c.keep_status("compact", pages={field: FAKE + 8}) == ALIGN
    for n in (0, -1, 2 ** 31):
        assert c.keep_status("compact", pages={"n_pages": n}) == SHAPE
    assert c.keep_status("compact", max_keep=-1) == SHAPE and c.keep_status("compact", max_keep=2 ** 31) == SHAPE
    assert c.keep_status("compact", per_head=2) == SHAPE and c.keep_status("compact", first=FAKE + 2) == ALIGN
    assert c.keep_status("compact", max_keep=0) == 0
    many = Call(heads=4096, kv_heads=4096, dim=16)
    assert many.keep_status("compact", batch={"n_seqs": 2 ** 20, "max_pages": 1}) == SHAPE


def test_binding_checks_tensors():
    ctx = make()
    pages, batch = cache(ctx)
    i32 = torch.int32
    q, lse, scores = torch.zeros(3, 4, 32), torch.zeros(3, 4), torch.zeros(3, 2, 8)
    masks, parents, keep, lens = torch.zeros(3, 1, dtype=torch.int64), torch.zeros(3, dtype=i32), torch.zeros(2, 2, 5, dtype=i32), torch.zeros(2, dtype=i32)
    good = {"masks": lambda **k: ctx.moe_tree_masks(**{"parents": parents, "batch": batch, **k}),
            "tree": lambda **k: ctx.moe_tree_attention(**{"q": q, "pages": pages, "batch": batch, "masks": masks, **k}),
            "weights": lambda **k: ctx.moe_kv_weights(**{"q": q, "lse": lse, "pages": pages, "batch": batch, "scores": scores, **k}),
            "select": lambda **k: ctx.moe_kv_select(**{"scores": scores, "batch": batch, "budget": 5, **k}),
            "compact": lambda **k: ctx.moe_kv_compact(**{"pages": pages, "batch": batch, "keep": keep, "keep_lens": lens, **k})}
    for f in good.values():
        with pytest.raises(ValueError, match="the kernels run on a GPU"):
            f()
    for name, bad in (("masks", {"parents": parents.long()}), ("masks", {"masks": masks.int()}), ("masks", {"words": 2, "masks": masks}),
                      ("masks", {"positions": parents[:2]}), ("masks", {"window": 2 ** 40}), ("masks", {"batch": None}),
                      ("tree", {"masks": masks[:2]}), ("tree", {"masks": masks[:, 0]}), ("tree", {"positions": lens}), ("tree", {"q": q[:, :2]}),
                      ("tree", {"sinks": torch.zeros(3)}), ("tree", {"lse": torch.zeros(3, 2)}), ("tree", {"pages": None}),
                      ("weights", {"lse": lse[:2]}), ("weights", {"scores": scores[:2]}), ("weights", {"scores": scores.double()}),
                      ("weights", {"q": q.bfloat16()}), ("weights", {"window": -2 ** 40}), ("select", {"scores": scores[:, :1]}),
                      ("select", {"keep": keep[:, :1]}), ("select", {"keep_lens": lens.long()}), ("select", {"budget": 2 ** 33}),
                      ("select", {"batch": binding.CKVBatch()}), ("compact", {"keep": keep.long()}), ("compact", {"keep": keep[:, 0, 0]}),
                      ("compact", {"keep": keep[:1]}), ("compact", {"keep_lens": lens[:1]}), ("compact", {"first": parents}),
                      ("compact", {"scores": scores[:1]}), ("compact", {"pages": binding.KVPages()})):
        with pytest.raises(ValueError) as e:
            good[name](**bad)
        assert "run on a GPU" not in str(e.value), (name, bad)
