"""Host-side checks of the key/value cache's entry points (no GPU): bad arguments are refused before any launch."""
import ctypes

import pytest
import torch

from paper_2510_08055_amd import binding

NULL, SHAPE, DTYPE, ALIGN, WORKSPACE = 1, 2, 3, 4, 5
FAKE = 0x10000       # never dereferenced: every call below fails a check first, or has no rows


def _cfg(heads=8, kv_heads=2, dim=64, page=16, dtype=1, fmt=0):
    return binding.CKVConfig(heads, kv_heads, dim, page, dtype, fmt)


def _bytes(**kw):
    n = ctypes.c_size_t(0)
    return binding.load().moe_kv_workspace_bytes(ctypes.byref(_cfg(**kw)), ctypes.byref(n)), n.value


def test_configurations():
    st, n = _bytes()
    assert st == 0 and n > 0
    assert _bytes(dim=256)[1] > n and binding.kv_workspace_bytes(8, 2, 64, 16, torch.bfloat16) == n
    for bad in ({"heads": 0}, {"kv_heads": 0}, {"kv_heads": 3}, {"heads": 8192, "kv_heads": 1}, {"dim": 0}, {"dim": 272}, {"page": 4},
                {"page": 24}, {"page": 512}, {"page": -16}):
        assert _bytes(**bad)[0] == SHAPE, bad
    assert _bytes(dim=72)[0] == ALIGN and _bytes(dim=8)[0] == ALIGN
    assert _bytes(dtype=2)[0] == DTYPE and _bytes(fmt=2)[0] == DTYPE and _bytes(fmt=-1)[0] == DTYPE
    lib, n = binding.load(), ctypes.c_size_t(0)
    assert lib.moe_kv_workspace_bytes(None, ctypes.byref(n)) == NULL
    assert lib.moe_kv_workspace_bytes(ctypes.byref(_cfg()), None) == NULL


def test_create():
    lib, ctx = binding.load(), ctypes.c_void_p()
    n = _bytes()[1]
    assert lib.moe_kv_create(ctypes.byref(_cfg()), None, n, ctypes.byref(ctx)) == NULL
    assert lib.moe_kv_create(ctypes.byref(_cfg()), FAKE, n, None) == NULL
    assert lib.moe_kv_create(ctypes.byref(_cfg()), FAKE, n - 1, ctypes.byref(ctx)) == WORKSPACE
    assert lib.moe_kv_create(ctypes.byref(_cfg()), FAKE + 128, n, ctypes.byref(ctx)) == ALIGN
    assert lib.moe_kv_create(ctypes.byref(_cfg(dim=20)), FAKE, n, ctypes.byref(ctx)) == ALIGN
    assert lib.moe_kv_destroy(None) == NULL


class Call:
    """The three calls with legal arguments but for what a test changes."""

    def __init__(self, **cfg):
        self.lib, self.ctx = binding.load(), ctypes.c_void_p()
        self.cfg = _cfg(**cfg)
        n = ctypes.c_size_t(0)
        assert self.lib.moe_kv_workspace_bytes(ctypes.byref(self.cfg), ctypes.byref(n)) == 0
        assert self.lib.moe_kv_create(ctypes.byref(self.cfg), FAKE, n, ctypes.byref(self.ctx)) == 0

    def status(self, what, T=4, pages=None, batch=None, q=FAKE, ldq=None, kv=FAKE, ldkv=None, out=FAKE, causal=1, window=0, sinks=None,
               lse=None, ctx=True):
        p = binding.CKVPages(FAKE, FAKE, FAKE, FAKE, 10)
        b = binding.CKVBatch(FAKE, FAKE, FAKE, 2, 8)
        for k, v in (pages or {}).items():
            setattr(p, k, v)
        for k, v in (batch or {}).items():
            setattr(b, k, v)
        c = self.ctx if ctx else None
        ldq = self.cfg.heads * self.cfg.dim if ldq is None else ldq
        ldkv = self.cfg.kv_heads * self.cfg.dim if ldkv is None else ldkv
        if what == "append":
            return self.lib.moe_kv_append(c, kv, ldkv, kv, ldkv, T, p, b, None)
        if what == "gather":
            return self.lib.moe_kv_gather(c, p, b, T, kv, ldkv, kv, ldkv, None)
        return self.lib.moe_paged_attention(c, q, ldq, T, p, b, binding.CAttentionOptions(causal, window, sinks), out, ldq, lse, None)


@pytest.mark.parametrize("what", ["append", "gather", "attention"])
def test_calls_refuse_bad_arguments(what):
    c = Call(fmt=1)
    assert c.status(what, T=0) == 0                                   # no rows: a no-op
    assert c.status(what, T=0, batch={"row_offsets": None, "n_seqs": 0, "max_pages": 0}) == 0
    assert c.status(what, ctx=False) == NULL
    assert c.status(what, T=-1) == SHAPE and c.status(what, T=2 ** 40) == SHAPE and c.status(what, T=2 ** 31) == SHAPE
    for field in ("k_pages", "v_pages", "k_scales", "v_scales"):
        assert c.status(what, pages={field: None}) == NULL, field
        assert c.status(what, pages={field: FAKE + 8}) == ALIGN, field
    for n in (0, -1, 2 ** 31):
        assert c.status(what, pages={"n_pages": n}) == SHAPE
    for field in ("row_offsets", "kv_lens", "page_table"):
        assert c.status(what, batch={field: None}) == NULL, field
        assert c.status(what, batch={field: FAKE + 2}) == ALIGN, field
    assert c.status(what, batch={"n_seqs": 0}) == SHAPE and c.status(what, batch={"n_seqs": -1}) == SHAPE
    assert c.status(what, batch={"max_pages": -1}) == SHAPE and c.status(what, batch={"max_pages": 2 ** 31}) == SHAPE
    if what == "attention":
        assert c.status(what, q=None) == NULL and c.status(what, out=None) == NULL
        assert c.status(what, q=FAKE + 8) == ALIGN and c.status(what, out=FAKE + 2) == ALIGN
        assert c.status(what, ldq=511) == SHAPE and c.status(what, ldq=516) == ALIGN
        assert c.status(what, causal=2) == SHAPE and c.status(what, window=-1) == SHAPE and c.status(what, window=2 ** 31 - 1) == SHAPE
        assert c.status(what, sinks=FAKE + 1) == ALIGN and c.status(what, lse=FAKE + 2) == ALIGN
    else:
        assert c.status(what, kv=None) == NULL and c.status(what, kv=FAKE + 8) == ALIGN
        assert c.status(what, ldkv=120) == SHAPE and c.status(what, ldkv=132) == ALIGN


def test_binding_checks_tensors():
    ctx = binding.KVContext(4, 2, 32, 8, torch.float32, device="cpu")
    pages = torch.zeros(3, 2, 8, 32)
    p = ctx.pack_pages(pages, pages.clone())
    with pytest.raises(ValueError):
        ctx.pack_pages(pages, pages[:2])
    with pytest.raises(ValueError):
        ctx.pack_pages(pages.bfloat16(), pages.bfloat16())
    with pytest.raises(ValueError):
        ctx.pack_pages(pages, pages, torch.zeros(3, 2, 8, dtype=torch.uint8), torch.zeros(3, 2, 8, dtype=torch.uint8))
    with pytest.raises(ValueError):
        binding.KVContext(4, 2, 32, 8, torch.float32, kv_format="fp8", device="cpu").pack_pages(pages.to(torch.float8_e4m3fn), pages.to(torch.float8_e4m3fn))
    off, lens, table = torch.tensor([0, 1, 3], dtype=torch.int32), torch.tensor([4, 5], dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32)
    b = ctx.pack_batch(off, lens, table)
    with pytest.raises(ValueError):
        ctx.pack_batch(off.long(), lens, table)
    with pytest.raises(ValueError):
        ctx.pack_batch(off[:2], lens, table)
    with pytest.raises(ValueError):
        ctx.pack_batch(off, lens, table[:1])
    q = torch.zeros(3, 4, 32)
    for bad in (q[:, :2], q.bfloat16(), torch.zeros(3, 32, 4).transpose(1, 2), torch.zeros(3, 8, 32)[:, ::2]):
        with pytest.raises(ValueError):
            ctx.moe_paged_attention(bad, p, b)
    with pytest.raises(ValueError):
        ctx.moe_paged_attention(q, p, b, sinks=torch.zeros(3))
    with pytest.raises(ValueError):
        ctx.moe_paged_attention(q, p, b, lse=torch.zeros(3, 2))
    with pytest.raises(ValueError):
        ctx.moe_kv_append(q[:, :2], q[:2, :2], p, b)
    with pytest.raises(TypeError):
        binding.KVContext(4, 2, 32, 8, torch.float16, device="cpu")
