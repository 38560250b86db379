// C ABI of the paged key/value cache and its attention: argument checks and workspace.  The arithmetic happens in the kernels of
// kv_cache.hip and attention.hip.
#include <cmath>
#include <new>

#include "kv.h"

using namespace moe;

struct moe_kv_ctx {
    moe_kv_config cfg;
    float* part;
    float2* part_stats;
    uint32_t* tickets;
    bool tickets_clear;
};

namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kMaxInt = 0x7fffffff;

moe_status check_cfg(const moe_kv_config* c)
{
    if (!c) return MOE_ERR_NULL;
    if (c->dtype != MOE_F32 && c->dtype != MOE_BF16) return MOE_ERR_DTYPE;
    if (c->kv_format != MOE_KV_DTYPE && c->kv_format != MOE_KV_FP8) return MOE_ERR_DTYPE;
    if (c->heads <= 0 || c->kv_heads <= 0 || c->heads % c->kv_heads || c->heads > 4096) return MOE_ERR_SHAPE;
    if (c->dim <= 0 || c->dim > 256 || c->page < 8 || c->page > 256 || (c->page & (c->page - 1))) return MOE_ERR_SHAPE;
    if (c->dim % 16) return MOE_ERR_ALIGN;
    return MOE_OK;
}

inline size_t part_bytes(const moe_kv_config& c) { return (size_t)kPartUnits * 16 * c.dim * sizeof(float); }
inline size_t stats_bytes() { return (size_t)kPartUnits * 16 * sizeof(float2); }
inline size_t workspace_size(const moe_kv_config& c) { return part_bytes(c) + stats_bytes() + kPartUnits * sizeof(uint32_t); }

inline bool misaligned(const void* p, uintptr_t to = 16) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
inline moe_status dev(hipError_t e) { return e == hipSuccess ? MOE_OK : e == hipErrorInvalidConfiguration ? MOE_ERR_SHAPE : MOE_ERR_DEVICE; }

// Rows of a tensor: `width` elements, ld apart, 16-byte aligned.
moe_status check_rows(const moe_kv_config& g, const void* p, int64_t ld, int64_t width)
{
    if (!p) return MOE_ERR_NULL;
    if (ld < width) return MOE_ERR_SHAPE;
    if (misaligned(p) || ld % (g.dtype == MOE_BF16 ? 8 : 4)) return MOE_ERR_ALIGN;
    return MOE_OK;
}

// The pages and the batch, as the kernels take them.
moe_status view_of(const moe_kv_ctx* ctx, const moe_kv_pages* pages, const moe_kv_batch* batch, int64_t T, KVView* out)
{
    if (!pages || !batch) return MOE_ERR_NULL;
    const moe_kv_config& g = ctx->cfg;
    if (T < 0 || batch->n_seqs < 0 || batch->max_pages < 0) return MOE_ERR_SHAPE;
    if (T > ((int64_t)1 << 30) / g.heads) return MOE_ERR_SHAPE;      // rows of heads are counted in 32 bits
    if (T > 0) {
        if (!pages->k_pages || !pages->v_pages || !batch->row_offsets || !batch->kv_lens) return MOE_ERR_NULL;
        if (batch->max_pages > 0 && !batch->page_table) return MOE_ERR_NULL;
        if (g.kv_format == MOE_KV_FP8 && (!pages->k_scales || !pages->v_scales)) return MOE_ERR_NULL;
        if (pages->n_pages < 1 || pages->n_pages > kMaxInt || batch->n_seqs < 1 || batch->n_seqs > kMaxInt / 512 ||
            batch->max_pages > ((int64_t)1 << 30) / g.page)
            return MOE_ERR_SHAPE;
        if (misaligned(pages->k_pages) || misaligned(pages->v_pages) || misaligned(pages->k_scales) || misaligned(pages->v_scales))
            return MOE_ERR_ALIGN;
        if (misaligned(batch->row_offsets, 4) || misaligned(batch->kv_lens, 4) || misaligned(batch->page_table, 4)) return MOE_ERR_ALIGN;
    }
    KVView& c = *out;
    c.k = static_cast<char*>(pages->k_pages);
    c.v = static_cast<char*>(pages->v_pages);
    c.ks = pages->k_scales;
    c.vs = pages->v_scales;
    c.off = batch->row_offsets;
    c.lens = batch->kv_lens;
    c.table = batch->page_table;
    c.n_pages = (int)pages->n_pages;
    c.S = (int)batch->n_seqs;
    c.max_pages = (int)batch->max_pages;
    c.T = (int)T;
    c.Hk = g.kv_heads;
    c.D = g.dim;
    c.page_shift = __builtin_ctz((unsigned)g.page);
    return MOE_OK;
}

}  // namespace

extern "C" {

moe_status moe_kv_workspace_bytes(const moe_kv_config* cfg, size_t* out_bytes)
{
    if (!out_bytes) return MOE_ERR_NULL;
    const moe_status st = check_cfg(cfg);
    if (st != MOE_OK) return st;
    *out_bytes = workspace_size(*cfg);
    return MOE_OK;
}

moe_status moe_kv_create(const moe_kv_config* cfg, void* workspace, size_t workspace_bytes, moe_kv_ctx** out_ctx)
{
    if (!out_ctx || !workspace) return MOE_ERR_NULL;
    const moe_status st = check_cfg(cfg);
    if (st != MOE_OK) return st;
    if (reinterpret_cast<uintptr_t>(workspace) % kAlign) return MOE_ERR_ALIGN;
    if (workspace_bytes < workspace_size(*cfg)) return MOE_ERR_WORKSPACE;
    moe_kv_ctx* c = new (std::nothrow) moe_kv_ctx();
    if (!c) return MOE_ERR_DEVICE;
    c->cfg = *cfg;
    c->part = static_cast<float*>(workspace);
    c->part_stats = reinterpret_cast<float2*>(static_cast<char*>(workspace) + part_bytes(*cfg));
    c->tickets = reinterpret_cast<uint32_t*>(static_cast<char*>(workspace) + part_bytes(*cfg) + stats_bytes());
    c->tickets_clear = false;
    *out_ctx = c;
    return MOE_OK;
}

moe_status moe_kv_destroy(moe_kv_ctx* ctx)
{
    if (!ctx) return MOE_ERR_NULL;
    delete ctx;
    return MOE_OK;
}

moe_status moe_kv_append(moe_kv_ctx* ctx, const void* k, int64_t ldk, const void* v, int64_t ldv, int64_t T, const moe_kv_pages* pages,
                         const moe_kv_batch* batch, void* stream)
{
    if (!ctx) return MOE_ERR_NULL;
    KVView c;
    moe_status st = view_of(ctx, pages, batch, T, &c);
    if (st != MOE_OK || T == 0) return st;
    const int64_t width = (int64_t)c.Hk * c.D;
    if ((st = check_rows(ctx->cfg, k, ldk, width)) != MOE_OK || (st = check_rows(ctx->cfg, v, ldv, width)) != MOE_OK) return st;
    return dev(launch_kv_append(ctx->cfg.dtype, ctx->cfg.kv_format == MOE_KV_FP8, c, k, ldk, v, ldv, static_cast<hipStream_t>(stream)));
}

moe_status moe_kv_gather(moe_kv_ctx* ctx, const moe_kv_pages* pages, const moe_kv_batch* batch, int64_t T, void* k, int64_t ldk, void* v,
                         int64_t ldv, void* stream)
{
    if (!ctx) return MOE_ERR_NULL;
    KVView c;
    moe_status st = view_of(ctx, pages, batch, T, &c);
    if (st != MOE_OK || T == 0) return st;
    const int64_t width = (int64_t)c.Hk * c.D;
    if ((st = check_rows(ctx->cfg, k, ldk, width)) != MOE_OK || (st = check_rows(ctx->cfg, v, ldv, width)) != MOE_OK) return st;
    return dev(launch_kv_gather(ctx->cfg.dtype, ctx->cfg.kv_format == MOE_KV_FP8, c, k, ldk, v, ldv, static_cast<hipStream_t>(stream)));
}

moe_status moe_paged_attention(moe_kv_ctx* ctx, const void* q, int64_t ldq, int64_t T, const moe_kv_pages* pages, const moe_kv_batch* batch,
                               const moe_attention_options* opt, void* out, int64_t ldo, float* lse, void* stream)
{
    if (!ctx || !opt) return MOE_ERR_NULL;
    AttnArgs a;
    moe_status st = view_of(ctx, pages, batch, T, &a.c);
    if (st != MOE_OK) return st;
    if ((opt->causal != 0 && opt->causal != 1) || opt->window < 0 || opt->window > 1 << 30) return MOE_ERR_SHAPE;
    if (T == 0) return MOE_OK;
    const moe_kv_config& g = ctx->cfg;
    const int64_t width = (int64_t)g.heads * g.dim;
    if ((st = check_rows(g, q, ldq, width)) != MOE_OK || (st = check_rows(g, out, ldo, width)) != MOE_OK) return st;
    if (misaligned(opt->sinks, 4) || misaligned(lse, 4)) return MOE_ERR_ALIGN;
    a.q = q;
    a.out = out;
    a.lse = lse;
    a.sinks = opt->sinks;
    a.ldq = ldq;
    a.ldo = ldo;
    a.Hq = g.heads;
    a.G = g.heads / g.kv_heads;
    a.causal = opt->causal;
    a.window = opt->window;
    a.scale2 = (float)(1.4426950408889634 / std::sqrt((double)g.dim));
    a.part = ctx->part;
    a.part_stats = ctx->part_stats;
    a.tickets = ctx->tickets;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    // The tickets are zero between launches once they have been cleared: in front of a context's first call.  A call that is
    // being captured carries the clear along, runs when its graph is replayed, and so leaves it to the next call as well.
    const bool clear = !ctx->tickets_clear;
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (clear && hipStreamIsCapturing(s, &capture) != hipSuccess) {
        (void)hipGetLastError();        // (the legacy stream while another one is captured)
        capture = hipStreamCaptureStatusActive;
    }
    st = dev(launch_attention(g.dtype, g.kv_format == MOE_KV_FP8, a, clear, s));
    if (clear) ctx->tickets_clear = st == MOE_OK && capture == hipStreamCaptureStatusNone;
    return st;
}

}  // extern "C"
