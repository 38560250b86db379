"""Thin ctypes binding over libmoe_lp.so (the C ABI declared in include/moe_lp.h).

Argument marshalling only: torch tensors supply device pointers and the current HIP
stream; every step of the path runs in the library's kernels.  There is no CPU
fallback: if the library is missing, `load()` raises.
"""
import ctypes
import os
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoe_lp.so")
_lib = None

MOE_F32, MOE_BF16 = 0, 1
MOE_SCHED_CHUNKED, MOE_SCHED_LAYERED = 0, 1
MOE_W_DTYPE, MOE_W_MXFP4 = 0, 1
MOE_KV_DTYPE, MOE_KV_FP8 = 0, 1
KV_FORMATS = {"": MOE_KV_DTYPE, "dtype": MOE_KV_DTYPE, "fp8": MOE_KV_FP8}
WEIGHT_FORMATS = {"": MOE_W_DTYPE, "dtype": MOE_W_DTYPE, "mxfp4": MOE_W_MXFP4}

EXPORTS = ["moe_workspace_bytes", "moe_create", "moe_destroy", "moe_router_topk", "moe_router_topk_noalloc", "moe_permute",
           "moe_grouped_ffn", "moe_grouped_ffn_mxfp4", "moe_combine", "moe_group_forward", "moe_num_layer_groups", "moe_layer_groups",
           "moe_stack_forward", "moe_read_counters", "moe_reset_counters",
           "moe_kernel_timing", "moe_read_kernel_timing", "moe_ffn_variant", "moe_set_ffn_variant",
           "moe_status_string", "moe_kv_workspace_bytes", "moe_kv_create", "moe_kv_destroy", "moe_kv_append", "moe_kv_gather",
           "moe_paged_attention"]

FFN_VARIANTS = {"auto": 0, "tile128": 1, "small": 2, "big": 3, "w4_tile64": 4, "w4_stream": 5, "w4_big": 6, "few": 7, "wide": 8}

KERNELS = {"router_logits": 0, "topk": 1, "permute": 2, "gate_up": 3, "down": 4, "combine": 5}


class MoeError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: moe_status {status} ({status_string(status)})")


class CConfig(ctypes.Structure):
    _fields_ = [("H", ctypes.c_int32), ("E", ctypes.c_int32), ("K", ctypes.c_int32), ("I", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("renormalize", ctypes.c_int32), ("residual", ctypes.c_int32),
                ("weight_format", ctypes.c_int32), ("y_perm_f32", ctypes.c_int32),
                ("act_split", ctypes.c_int32)]


class CLayer(ctypes.Structure):
    _fields_ = [("w_router", ctypes.c_void_p), ("router_bias", ctypes.c_void_p),
                ("w_gate_up", ctypes.c_void_p), ("w_down", ctypes.c_void_p),
                ("s_gate_up", ctypes.c_void_p), ("s_down", ctypes.c_void_p)]


class CSchedule(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("chunk", ctypes.c_int32)]


class CStackSchedule(ctypes.Structure):
    _fields_ = [("chunk", ctypes.c_int32), ("n_groups", ctypes.c_int32), ("granule", ctypes.c_int32)]


class CCounters(ctypes.Structure):
    _fields_ = [("expert_bytes", ctypes.c_uint64), ("router_bytes", ctypes.c_uint64),
                ("active_experts_total", ctypes.c_uint64), ("tokens_processed", ctypes.c_uint64),
                ("iterations", ctypes.c_uint32), ("layer_passes", ctypes.c_uint32)]


class CKVConfig(ctypes.Structure):
    _fields_ = [("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("dim", ctypes.c_int32), ("page", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("kv_format", ctypes.c_int32)]


class CKVPages(ctypes.Structure):
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p), ("k_scales", ctypes.c_void_p),
                ("v_scales", ctypes.c_void_p), ("n_pages", ctypes.c_int64)]


class CKVBatch(ctypes.Structure):
    _fields_ = [("row_offsets", ctypes.c_void_p), ("kv_lens", ctypes.c_void_p), ("page_table", ctypes.c_void_p),
                ("n_seqs", ctypes.c_int64), ("max_pages", ctypes.c_int64)]


class CAttentionOptions(ctypes.Structure):
    _fields_ = [("causal", ctypes.c_int32), ("window", ctypes.c_int32), ("sinks", ctypes.c_void_p)]


@dataclass
class Counters:
    expert_bytes: int
    router_bytes: int
    active_experts_total: int
    tokens_processed: int
    iterations: int
    layer_passes: int


def load():
    """Load the C-ABI library; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                           "(or paper_2510_08055_amd/build.py); the HIP library is required")
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
    L.moe_workspace_bytes.argtypes = [ctypes.POINTER(CConfig), i64, ctypes.POINTER(ctypes.c_size_t)]
    L.moe_create.argtypes = [ctypes.POINTER(CConfig), i64, vp, ctypes.c_size_t, vp, ctypes.POINTER(vp)]
    L.moe_destroy.argtypes = [vp]
    L.moe_router_topk.argtypes = [vp, vp, i64, vp, vp, vp, vp, vp]
    L.moe_router_topk_noalloc.argtypes = [ctypes.POINTER(CConfig), vp, i64, vp, vp, vp, vp, vp]
    L.moe_permute.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, vp, vp]
    L.moe_grouped_ffn.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp]
    L.moe_grouped_ffn_mxfp4.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, vp, vp]
    L.moe_combine.argtypes = [vp, vp, vp, vp, vp, i64, vp, vp]
    L.moe_group_forward.argtypes = [vp, ctypes.POINTER(CLayer), i32, vp, i64, vp, i64, CSchedule, vp, vp, vp]
    L.moe_num_layer_groups.argtypes = [i64, i32, i32]
    L.moe_layer_groups.argtypes = [i32, i32, ctypes.POINTER(i32)]
    L.moe_stack_forward.argtypes = [vp, ctypes.POINTER(CLayer), i32, vp, i64, vp, i64, CStackSchedule, vp, vp, vp]
    L.moe_read_counters.argtypes = [vp, ctypes.POINTER(CCounters), vp]
    L.moe_reset_counters.argtypes = [vp, vp]
    L.moe_kernel_timing.argtypes = [vp, ctypes.c_uint32]
    L.moe_read_kernel_timing.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i64), vp]
    L.moe_ffn_variant.argtypes = [vp, i64]
    L.moe_ffn_variant.restype = ctypes.c_char_p
    L.moe_set_ffn_variant.argtypes = [vp, i32]
    pages, batch = ctypes.POINTER(CKVPages), ctypes.POINTER(CKVBatch)
    L.moe_kv_workspace_bytes.argtypes = [ctypes.POINTER(CKVConfig), ctypes.POINTER(ctypes.c_size_t)]
    L.moe_kv_create.argtypes = [ctypes.POINTER(CKVConfig), vp, ctypes.c_size_t, ctypes.POINTER(vp)]
    L.moe_kv_destroy.argtypes = [vp]
    L.moe_kv_append.argtypes = [vp, vp, i64, vp, i64, i64, pages, batch, vp]
    L.moe_kv_gather.argtypes = [vp, pages, batch, i64, vp, i64, vp, i64, vp]
    L.moe_paged_attention.argtypes = [vp, vp, i64, i64, pages, batch, ctypes.POINTER(CAttentionOptions), vp, i64, vp, vp]
    L.moe_status_string.argtypes = [i32]
    L.moe_status_string.restype = ctypes.c_char_p
    for name in EXPORTS:
        if name not in ("moe_ffn_variant", "moe_status_string"):
            getattr(L, name).restype = ctypes.c_int       # moe_status, or a count for moe_num_layer_groups
    _lib = L
    return L


def status_string(status: int) -> str:
    return load().moe_status_string(int(status)).decode()


def _check(status: int, what: str):
    if status != 0:
        raise MoeError(status, what)


def moe_num_layer_groups(prompt_len: int, n_layers: int, granule: int = 512) -> int:
    """N_lg(L) = max(1, ceil(L / granule)), at most n_layers; 0 for invalid arguments (host arithmetic)."""
    return int(load().moe_num_layer_groups(int(prompt_len), int(n_layers), int(granule)))


def moe_layer_groups(n_layers: int, n_groups: int):
    """first_layer[0..n_groups]: group g holds layers first_layer[g] .. first_layer[g+1]-1."""
    out = (ctypes.c_int32 * (max(int(n_groups), 0) + 1))()
    _check(load().moe_layer_groups(int(n_layers), int(n_groups), out), "moe_layer_groups")
    return list(out)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_contiguous(), "tensors handed to the C ABI must be contiguous"
    return ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.bfloat16:
        return MOE_BF16
    if dt == torch.float32:
        return MOE_F32
    raise TypeError(f"unsupported dtype {dt}")


def workspace_bytes(H, E, K, I, dtype, max_tokens, renormalize=True, residual=True, weight_format="",
                    y_perm_f32=False, act_split=False) -> int:
    cfg = CConfig(H, E, K, I, _dtype_code(dtype), int(renormalize), int(residual), WEIGHT_FORMATS[weight_format],
                  int(y_perm_f32), int(act_split))
    out = ctypes.c_size_t(0)
    _check(load().moe_workspace_bytes(ctypes.byref(cfg), max_tokens, ctypes.byref(out)), "moe_workspace_bytes")
    return out.value


def moe_router_topk_noalloc(x, w_router, bias, K, renormalize=True, topk_idx=None, topk_w=None):
    """The router without a context or workspace (the library's static scratch holds the logits).  The outputs
    may be passed in, so that the call itself allocates nothing."""
    T, H = x.shape
    E = w_router.shape[0]
    cfg = CConfig(H, E, K, 8, _dtype_code(x.dtype), int(renormalize), 0, MOE_W_DTYPE, 0, 0)
    if topk_idx is None:
        topk_idx = torch.empty((T, K), dtype=torch.int32, device=x.device)
    if topk_w is None:
        topk_w = torch.empty((T, K), dtype=torch.float32, device=x.device)
    with torch.cuda.device(x.device):
        _check(load().moe_router_topk_noalloc(ctypes.byref(cfg), _ptr(x), T, _ptr(w_router), _ptr(bias), _ptr(topk_idx),
                                              _ptr(topk_w), _stream()), "moe_router_topk_noalloc")
    return topk_idx, topk_w


class Context:
    """A moe_ctx plus the torch-allocated workspace it lives on."""

    def __init__(self, H, E, K, I, dtype=torch.bfloat16, max_tokens=1024, renormalize=True, residual=True,
                 device="cuda:0", weight_format="", y_perm_f32=False, act_split=False):
        self.lib = load()
        self.H, self.E, self.K, self.I = H, E, K, I
        self.dtype = dtype
        self.max_tokens = max_tokens
        self.device = torch.device(device)
        self.weight_format = weight_format
        self.y_perm_dtype = torch.float32 if y_perm_f32 else dtype
        self.cfg = CConfig(H, E, K, I, _dtype_code(dtype), int(renormalize), int(residual),
                           WEIGHT_FORMATS[weight_format], int(y_perm_f32), int(act_split))
        n = ctypes.c_size_t(0)
        _check(self.lib.moe_workspace_bytes(ctypes.byref(self.cfg), max_tokens, ctypes.byref(n)),
               "moe_workspace_bytes")
        self.workspace = torch.empty(n.value + 256, dtype=torch.uint8, device=self.device)
        base = (self.workspace.data_ptr() + 255) // 256 * 256
        self._ctx = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check(self.lib.moe_create(ctypes.byref(self.cfg), max_tokens, ctypes.c_void_p(base), n.value, _stream(),
                                       ctypes.byref(self._ctx)), "moe_create")

    def close(self):
        if self._ctx:
            self.lib.moe_destroy(self._ctx)
            self._ctx = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- the five calls of the boundary, same names as the C ABI ----

    def moe_router_topk(self, x, w_router, bias=None):
        T = x.shape[0]
        idx = torch.empty((T, self.K), dtype=torch.int32, device=self.device)
        w = torch.empty((T, self.K), dtype=torch.float32, device=self.device)
        _check(self.lib.moe_router_topk(self._ctx, _ptr(x), T, _ptr(w_router), _ptr(bias), _ptr(idx), _ptr(w),
                                        _stream()), "moe_router_topk")
        return idx, w

    def moe_permute(self, x, topk_idx, want_x_perm=True):
        T = topk_idx.shape[0]
        A = T * self.K
        counts = torch.empty(self.E, dtype=torch.int32, device=self.device)
        offsets = torch.empty(self.E + 1, dtype=torch.int32, device=self.device)
        perm = torch.empty(A, dtype=torch.int32, device=self.device)
        inv = torch.empty(A, dtype=torch.int32, device=self.device)
        x_perm = torch.empty((A, self.H), dtype=self.dtype, device=self.device) if want_x_perm else None
        _check(self.lib.moe_permute(self._ctx, _ptr(x), _ptr(topk_idx), T, _ptr(counts), _ptr(offsets), _ptr(perm),
                                    _ptr(inv), _ptr(x_perm), _stream()), "moe_permute")
        return counts, offsets, perm, inv, x_perm

    def moe_grouped_ffn(self, x_perm, offsets, w_gate_up, w_down):
        A = x_perm.shape[0]
        y_perm = torch.empty((A, self.H), dtype=self.y_perm_dtype, device=self.device)
        _check(self.lib.moe_grouped_ffn(self._ctx, _ptr(x_perm), _ptr(offsets), A, _ptr(w_gate_up), _ptr(w_down),
                                        _ptr(y_perm), _stream()), "moe_grouped_ffn")
        return y_perm

    def moe_grouped_ffn_mxfp4(self, x_perm, offsets, w_gate_up, s_gate_up, w_down, s_down):
        A = x_perm.shape[0]
        y_perm = torch.empty((A, self.H), dtype=self.y_perm_dtype, device=self.device)
        _check(self.lib.moe_grouped_ffn_mxfp4(self._ctx, _ptr(x_perm), _ptr(offsets), A, _ptr(w_gate_up),
                                              _ptr(s_gate_up), _ptr(w_down), _ptr(s_down), _ptr(y_perm), _stream()),
               "moe_grouped_ffn_mxfp4")
        return y_perm

    def moe_combine(self, y_perm, inv_perm, topk_w, residual=None, out=None):
        T = topk_w.shape[0]
        y = out if out is not None else torch.empty((T, self.H), dtype=self.dtype, device=self.device)
        _check(self.lib.moe_combine(self._ctx, _ptr(y_perm), _ptr(inv_perm), _ptr(topk_w), _ptr(residual), T,
                                    _ptr(y), _stream()), "moe_combine")
        return y

    def pack_layers(self, layers: Sequence[dict]):
        """Host array of moe_layer structs from dicts of device tensors (kept alive by the caller)."""
        arr = (CLayer * len(layers))()
        for i, L in enumerate(layers):
            b = L.get("router_bias")
            sg, sd = L.get("s_gate_up"), L.get("s_down")
            arr[i] = CLayer(L["w_router"].data_ptr(), b.data_ptr() if b is not None else None,
                            L["w_gate_up"].data_ptr(), L["w_down"].data_ptr(),
                            sg.data_ptr() if sg is not None else None, sd.data_ptr() if sd is not None else None)
        return arr

    def moe_group_forward(self, layers, x_decode, x_prefill, schedule="layered", chunk=0, packed=None,
                          y_decode=None, y_prefill=None):
        D = 0 if x_decode is None else x_decode.shape[0]
        P = 0 if x_prefill is None else x_prefill.shape[0]
        arr = packed if packed is not None else self.pack_layers(layers)
        if y_decode is None:
            y_decode = torch.empty((D, self.H), dtype=self.dtype, device=self.device)
        if y_prefill is None:
            y_prefill = torch.empty((P, self.H), dtype=self.dtype, device=self.device)
        kind = {"chunked": MOE_SCHED_CHUNKED, "layered": MOE_SCHED_LAYERED}[schedule]
        _check(self.lib.moe_group_forward(self._ctx, arr, len(arr), _ptr(x_decode) if D else None, D,
                                          _ptr(x_prefill) if P else None, P, CSchedule(kind, int(chunk)),
                                          _ptr(y_decode) if D else None, _ptr(y_prefill) if P else None, _stream()),
               "moe_group_forward")
        return y_decode, y_prefill

    def moe_stack_forward(self, layers, x_decode, x_prefill, chunk=0, n_groups=0, granule=512, packed=None,
                          y_decode=None, y_prefill=None):
        D = 0 if x_decode is None else x_decode.shape[0]
        P = 0 if x_prefill is None else x_prefill.shape[0]
        arr = packed if packed is not None else self.pack_layers(layers)
        if y_decode is None:
            y_decode = torch.empty((D, self.H), dtype=self.dtype, device=self.device)
        if y_prefill is None:
            y_prefill = torch.empty((P, self.H), dtype=self.dtype, device=self.device)
        _check(self.lib.moe_stack_forward(self._ctx, arr, len(arr), _ptr(x_decode) if D else None, D,
                                          _ptr(x_prefill) if P else None, P,
                                          CStackSchedule(int(chunk), int(n_groups), int(granule)),
                                          _ptr(y_decode) if D else None, _ptr(y_prefill) if P else None, _stream()),
               "moe_stack_forward")
        return y_decode, y_prefill

    def moe_read_counters(self) -> Counters:
        c = CCounters()
        _check(self.lib.moe_read_counters(self._ctx, ctypes.byref(c), _stream()), "moe_read_counters")
        return Counters(c.expert_bytes, c.router_bytes, c.active_experts_total, c.tokens_processed, c.iterations,
                        c.layer_passes)

    def moe_reset_counters(self):
        _check(self.lib.moe_reset_counters(self._ctx, _stream()), "moe_reset_counters")

    def moe_kernel_timing(self, kernels=()):
        mask = 0
        for k in kernels:
            mask |= 1 << KERNELS[k]
        _check(self.lib.moe_kernel_timing(self._ctx, mask), "moe_kernel_timing")

    def moe_read_kernel_timing(self, kernel: str):
        """(total milliseconds, launches) of one timed kernel since moe_kernel_timing was set."""
        ms, n = ctypes.c_double(0), ctypes.c_int64(0)
        _check(self.lib.moe_read_kernel_timing(self._ctx, KERNELS[kernel], ctypes.byref(ms), ctypes.byref(n),
                                               _stream()), "moe_read_kernel_timing")
        return ms.value, n.value

    def moe_ffn_variant(self, T: int) -> str:
        return self.lib.moe_ffn_variant(self._ctx, T).decode()

    def moe_set_ffn_variant(self, variant="auto"):
        """Pin the grouped-GEMM kernel shape of this context (a name of FFN_VARIANTS, or the id)."""
        v = FFN_VARIANTS[variant] if isinstance(variant, str) else int(variant)
        _check(self.lib.moe_set_ffn_variant(self._ctx, v), "moe_set_ffn_variant")


def _int32(name, v):
    """ctypes would drop its upper bits without a word."""
    if not -0x80000000 <= v <= 0x7fffffff:
        raise ValueError(f"{name}: {v} does not fit 32 bits")
    return int(v)


def _kv_config(heads, kv_heads, dim, page, dtype, kv_format):
    return CKVConfig(_int32("heads", heads), _int32("kv_heads", kv_heads), _int32("dim", dim), _int32("page", page), _dtype_code(dtype),
                     KV_FORMATS[kv_format])


def kv_workspace_bytes(heads, kv_heads, dim, page, dtype, kv_format="") -> int:
    cfg = _kv_config(heads, kv_heads, dim, page, dtype, kv_format)
    out = ctypes.c_size_t(0)
    _check(load().moe_kv_workspace_bytes(ctypes.byref(cfg), ctypes.byref(out)), "moe_kv_workspace_bytes")
    return out.value


class KVPages(CKVPages):
    """The pages of one layer (moe_kv_pages); keeps their tensors alive, and the layout that they were checked for."""
    tensors = ()
    layout = None


class KVBatch(CKVBatch):
    """A batch's descriptors (moe_kv_batch); keeps their tensors alive."""
    tensors = ()
    device = None


_the_same = {}       # equal values as one object, so that a call compares identities


class KVContext:
    """A moe_kv_ctx plus the torch-allocated workspace it lives on: a paged key/value cache's format and its attention.

    Tensors of rows (q, k, v and what comes back) are [T, heads, dim] with any stride between rows, so views of one fused
    projection can be handed over.  The struct of a batch holds pointers only: what its tensors hold when a call runs counts.
    Contexts of the same layout (kv_heads, page, dim, the pages' type, the GPU) may share packed pages; others refuse them."""

    def __init__(self, heads, kv_heads, dim, page, dtype=torch.bfloat16, kv_format="", device="cuda:0"):
        self.lib = load()
        self.heads, self.kv_heads, self.dim, self.page = heads, kv_heads, dim, page
        self.dtype = dtype
        self.kv_format = kv_format
        self.device = torch.device(device)
        self.cfg = _kv_config(heads, kv_heads, dim, page, dtype, kv_format)
        self.fp8 = self.cfg.kv_format == MOE_KV_FP8
        self.page_dtype = torch.float8_e4m3fn if self.fp8 else dtype
        n = ctypes.c_size_t(0)
        _check(self.lib.moe_kv_workspace_bytes(ctypes.byref(self.cfg), ctypes.byref(n)), "moe_kv_workspace_bytes")
        self.workspace = torch.empty(n.value + 256, dtype=torch.uint8, device=self.device)
        layout = (kv_heads, page, dim, self.page_dtype, self.workspace.device)
        self.layout = _the_same.setdefault(layout, layout)
        self.batch_device = _the_same.setdefault(self.workspace.device, self.workspace.device)
        base = (self.workspace.data_ptr() + 255) // 256 * 256
        self._ctx = ctypes.c_void_p()
        _check(self.lib.moe_kv_create(ctypes.byref(self.cfg), ctypes.c_void_p(base), n.value, ctypes.byref(self._ctx)), "moe_kv_create")

    def close(self):
        if self._ctx:
            self.lib.moe_kv_destroy(self._ctx)
            self._ctx = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _call(self, name, *args):
        """A call of the library on the context's GPU and that GPU's current stream."""
        if self.device.type != "cuda":
            raise ValueError(f"the kernels run on a GPU, not on {self.device}")
        gpu = self.workspace.device.index
        if torch._C._cuda_getDevice() != gpu:
            with torch.cuda.device(gpu):
                return self._call(name, *args)
        # (the handle itself: torch.cuda.current_stream() takes 3 us to wrap it, as long as a launch)
        _check(getattr(self.lib, name)(self._ctx, *args, torch._C._cuda_getCurrentRawStream(gpu)), name)

    def _packed(self, pages, batch):
        """The structs hold pointers alone, so what pack_pages and pack_batch checked has to be what this context reads."""
        if getattr(pages, "layout", None) is not self.layout:
            raise ValueError(f"pages packed for {getattr(pages, 'layout', None)} do not belong to a context of {self.layout}")
        if getattr(batch, "device", None) is not self.batch_device:
            raise ValueError(f"a batch packed on {getattr(batch, 'device', None)} does not belong to a context on {self.batch_device}")

    def _dense(self, t, name, dtype, shape):
        if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous() or t.device != self.workspace.device:
            raise ValueError(f"{name}: a contiguous {dtype} tensor {shape} on {self.workspace.device} is needed, "
                             f"not {t.dtype} {tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    def _rows(self, t, name, T, heads):
        """Pointer and row stride of a [T, heads, dim] tensor."""
        if t.shape != (T, heads, self.dim) or t.dtype != self.dtype or t.device != self.workspace.device:
            raise ValueError(f"{name}: a {self.dtype} tensor {(T, heads, self.dim)} on {self.workspace.device} is needed, "
                             f"not {t.dtype} {tuple(t.shape)} on {t.device}")
        ld, head, one = t.stride()
        if (one != 1 and self.dim > 1) or (head != self.dim and heads > 1):
            raise ValueError(f"{name}: a row's heads must lie side by side, not with strides {t.stride()}")
        return t.data_ptr(), (ld if T > 1 else heads * self.dim)

    def pack_pages(self, k_pages, v_pages, k_scales=None, v_scales=None) -> KVPages:
        """The struct of a layer's pages [n_pages, kv_heads, page, dim] (and scales [n_pages, kv_heads, page] of FP8 ones)."""
        n = k_pages.shape[0]
        shape = (n, self.kv_heads, self.page, self.dim)
        p = KVPages(self._dense(k_pages, "k_pages", self.page_dtype, shape), self._dense(v_pages, "v_pages", self.page_dtype, shape),
                    None, None, n)
        if self.fp8:
            if k_scales is None or v_scales is None:
                raise ValueError("FP8 pages need k_scales and v_scales")
            p.k_scales = self._dense(k_scales, "k_scales", torch.uint8, shape[:3])
            p.v_scales = self._dense(v_scales, "v_scales", torch.uint8, shape[:3])
        elif k_scales is not None or v_scales is not None:
            raise ValueError("scales belong to FP8 pages")
        p.tensors = (k_pages, v_pages, k_scales, v_scales)
        p.layout = self.layout
        return p

    def pack_batch(self, row_offsets, kv_lens, page_table) -> KVBatch:
        """The struct of a batch's descriptors: row_offsets [n_seqs + 1], kv_lens [n_seqs], page_table [n_seqs, max_pages], int32."""
        n = kv_lens.shape[0]
        b = KVBatch(self._dense(row_offsets, "row_offsets", torch.int32, (n + 1,)), self._dense(kv_lens, "kv_lens", torch.int32, (n,)),
                    self._dense(page_table, "page_table", torch.int32, (n, page_table.shape[1])), n, page_table.shape[1])
        b.tensors = (row_offsets, kv_lens, page_table)
        b.device = self.batch_device
        return b

    # ---- the calls of the boundary, same names as the C ABI ----

    def moe_kv_append(self, k, v, pages, batch):
        self._packed(pages, batch)
        T = k.shape[0]
        kp, ldk = self._rows(k, "k", T, self.kv_heads)
        vp, ldv = self._rows(v, "v", T, self.kv_heads)
        self._call("moe_kv_append", kp, ldk, vp, ldv, T, pages, batch)

    def moe_kv_gather(self, pages, batch, T=None, k=None, v=None):
        """The rows' keys and values [T, kv_heads, dim]; T: the batch's rows, needed where no outputs are passed in."""
        self._packed(pages, batch)
        if k is None or v is None:
            T = T if T is not None else (k if k is not None else v).shape[0]
            made = [torch.empty((T, self.kv_heads, self.dim), dtype=self.dtype, device=self.device) for t in (k, v) if t is None]
            k = made.pop() if k is None else k
            v = made.pop() if v is None else v
        T = k.shape[0]
        kp, ldk = self._rows(k, "k", T, self.kv_heads)
        vp, ldv = self._rows(v, "v", T, self.kv_heads)
        self._call("moe_kv_gather", pages, batch, T, kp, ldk, vp, ldv)
        return k, v

    def moe_paged_attention(self, q, pages, batch, causal=True, window=0, sinks=None, out=None, lse=None):
        """out [T, heads, dim]; lse: a [T, heads] fp32 tensor to receive the rows' log-sum-exp, or None."""
        self._packed(pages, batch)
        T = q.shape[0]
        if out is None:
            out = torch.empty((T, self.heads, self.dim), dtype=self.dtype, device=self.device)
        qp, ldq = self._rows(q, "q", T, self.heads)
        op, ldo = self._rows(out, "out", T, self.heads)
        opt = CAttentionOptions(int(bool(causal)), _int32("window", window),
                                self._dense(sinks, "sinks", torch.float32, (self.heads,)) if sinks is not None else None)
        lp = self._dense(lse, "lse", torch.float32, (T, self.heads)) if lse is not None else None
        self._call("moe_paged_attention", qp, ldq, T, pages, batch, opt, op, ldo, lp)
        return out
