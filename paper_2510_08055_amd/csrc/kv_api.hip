// C ABI of the paged key/value cache and its attention: argument checks and workspace.  The arithmetic happens in the kernels of
// kv_cache.hip, attention.hip, tree_attention.hip, kv_tree.hip, kv_weights.hip, kv_select.hip and kv_compact.hip.
#include <cmath>
#include <new>

#include "kv.h"

using namespace moe;

struct moe_kv_ctx {
    moe_kv_config cfg;
    float* part;
    float2* part_stats;
    uint32_t *tickets, *compact_state;
    bool tickets_clear, compact_clear;      // (whether they are known to be zero)
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
inline size_t workspace_size(const moe_kv_config& c) { return part_bytes(c) + stats_bytes() + (kPartUnits + kCompactWords) * sizeof(uint32_t); }

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

// The descriptors of a call that takes no rows: lengths and page table.
moe_status view_of_tokens(const moe_kv_ctx* ctx, int64_t n_pages, const moe_kv_batch* batch, KVView* out)
{
    if (!batch) return MOE_ERR_NULL;
    const moe_kv_config& g = ctx->cfg;
    if (batch->n_seqs < 0 || batch->max_pages < 0) return MOE_ERR_SHAPE;
    if (batch->n_seqs > 0) {
        if (!batch->kv_lens || (batch->max_pages > 0 && !batch->page_table)) return MOE_ERR_NULL;
        if (n_pages < 1 || n_pages > kMaxInt || batch->n_seqs > kMaxInt / 512 || batch->max_pages > ((int64_t)1 << 30) / g.page) return MOE_ERR_SHAPE;
        if (misaligned(batch->kv_lens, 4) || misaligned(batch->page_table, 4)) return MOE_ERR_ALIGN;
    }
    *out = KVView{};
    out->lens = batch->kv_lens;
    out->table = batch->page_table;
    out->n_pages = (int)n_pages;
    out->S = (int)batch->n_seqs;
    out->max_pages = (int)batch->max_pages;
    out->Hk = g.kv_heads;
    out->D = g.dim;
    out->page_shift = __builtin_ctz((unsigned)g.page);
    return MOE_OK;
}

inline float scale2_of(const moe_kv_config& g) { return (float)(1.4426950408889634 / std::sqrt((double)g.dim)); }

// A launch that uses counters of the workspace.  They are zero between launches once they have been cleared (is_clear): in front of a context's first
// call.  A call that is being captured carries the clear along, runs when its graph is replayed, and so leaves it to the next call as well.
// (launch may say that it did not clear them: bool&.)
template <typename F> moe_status with_counters(bool& is_clear, void* stream, F launch)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    bool clear = !is_clear;
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (clear && hipStreamIsCapturing(s, &capture) != hipSuccess) {
        (void)hipGetLastError();        // (the legacy stream while another one is captured)
        capture = hipStreamCaptureStatusActive;
    }
    const moe_status st = dev(launch(clear, s));
    if (clear) is_clear = st == MOE_OK && capture == hipStreamCaptureStatusNone;
    return st;
}

// Attention, of rows as they follow each other or (tree) of trees.
moe_status attend(moe_kv_ctx* ctx, const void* q, int64_t ldq, int64_t T, const moe_kv_pages* pages, const moe_kv_batch* batch, const moe_tree* tree,
                  const moe_attention_options* opt, void* out, int64_t ldo, float* lse, void* stream)
{
    AttnArgs a;
    moe_status st = view_of(ctx, pages, batch, T, &a.c);
    if (st != MOE_OK) return st;
    if ((opt->causal != 0 && opt->causal != 1) || opt->window < 0 || opt->window > 1 << 30) return MOE_ERR_SHAPE;
    if (tree && (tree->words < 1 || tree->words > kMaxTreeWords || opt->causal != 1)) return MOE_ERR_SHAPE;
    if (T == 0) return MOE_OK;
    if (tree && (!tree->masks || (opt->window > 0 && !tree->positions))) return MOE_ERR_NULL;
    const moe_kv_config& g = ctx->cfg;
    const int64_t width = (int64_t)g.heads * g.dim;
    if ((st = check_rows(g, q, ldq, width)) != MOE_OK || (st = check_rows(g, out, ldo, width)) != MOE_OK) return st;
    if (misaligned(opt->sinks, 4) || misaligned(lse, 4)) return MOE_ERR_ALIGN;
    if (tree && (misaligned(tree->masks, 8) || misaligned(tree->positions, 4))) return MOE_ERR_ALIGN;
    a.q = q;
    a.out = out;
    a.lse = lse;
    a.sinks = opt->sinks;
    a.ldq = ldq;
    a.ldo = ldo;
    a.masks = tree ? tree->masks : nullptr;
    a.positions = tree ? tree->positions : nullptr;
    a.words = tree ? tree->words : 0;
    a.Hq = g.heads;
    a.G = g.heads / g.kv_heads;
    a.causal = opt->causal;
    a.window = opt->window;
    a.scale2 = scale2_of(g);
    a.part = ctx->part;
    a.part_stats = ctx->part_stats;
    a.tickets = ctx->tickets;
    return with_counters(ctx->tickets_clear, stream, [&](bool clear, hipStream_t s) {
        return tree ? launch_tree_attention(g.dtype, g.kv_format == MOE_KV_FP8, a, clear, s) : launch_attention(g.dtype, g.kv_format == MOE_KV_FP8, a, clear, s);
    });
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
    c->compact_state = c->tickets + kPartUnits;
    c->tickets_clear = c->compact_clear = false;
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
    return attend(ctx, q, ldq, T, pages, batch, nullptr, opt, out, ldo, lse, stream);
}

moe_status moe_tree_attention(moe_kv_ctx* ctx, const void* q, int64_t ldq, int64_t T, const moe_kv_pages* pages, const moe_kv_batch* batch,
                              const moe_tree* tree, const moe_attention_options* opt, void* out, int64_t ldo, float* lse, void* stream)
{
    if (!ctx || !tree || !opt) return MOE_ERR_NULL;
    return attend(ctx, q, ldq, T, pages, batch, tree, opt, out, ldo, lse, stream);
}

moe_status moe_tree_masks(moe_kv_ctx* ctx, const int32_t* parents, int64_t T, const moe_kv_batch* batch, int32_t words, int32_t window,
                          uint64_t* masks, int32_t* positions, void* stream)
{
    if (!ctx || !batch) return MOE_ERR_NULL;
    if (T < 0 || T > ((int64_t)1 << 30) / ctx->cfg.heads || words < 1 || words > kMaxTreeWords || window < 0 || window > 1 << 30) return MOE_ERR_SHAPE;
    if (T == 0) return batch->n_seqs < 0 ? MOE_ERR_SHAPE : MOE_OK;
    if (!parents || !masks || !batch->row_offsets || !batch->kv_lens) return MOE_ERR_NULL;
    if (batch->n_seqs < 1 || batch->n_seqs > kMaxInt / 512) return MOE_ERR_SHAPE;
    if (misaligned(parents, 4) || misaligned(masks, 8) || misaligned(positions, 4) || misaligned(batch->row_offsets, 4) ||
        misaligned(batch->kv_lens, 4))
        return MOE_ERR_ALIGN;
    KVView c = {};
    c.off = batch->row_offsets;
    c.lens = batch->kv_lens;
    c.S = (int)batch->n_seqs;
    c.T = (int)T;
    return dev(launch_tree_masks(c, parents, words, window, masks, positions, static_cast<hipStream_t>(stream)));
}

moe_status moe_kv_weights(moe_kv_ctx* ctx, const void* q, int64_t ldq, const float* lse, int64_t T, const moe_kv_pages* pages,
                          const moe_kv_batch* batch, const moe_weights_options* opt, float* scores, void* stream)
{
    if (!ctx || !opt) return MOE_ERR_NULL;
    WeightArgs a;
    moe_status st = view_of(ctx, pages, batch, T, &a.c);
    if (st != MOE_OK) return st;
    if ((opt->causal != 0 && opt->causal != 1) || opt->window < 0 || opt->window > 1 << 30 || !(opt->decay >= 0.0f && opt->decay <= 1.0f))
        return MOE_ERR_SHAPE;
    if (T == 0) return MOE_OK;
    if (ldq > 1 << 23) return MOE_ERR_SHAPE;      // (rows of a step lie within 2^31 bytes)
    if (!lse || !scores) return MOE_ERR_NULL;
    const moe_kv_config& g = ctx->cfg;
    if ((st = check_rows(g, q, ldq, (int64_t)g.heads * g.dim)) != MOE_OK) return st;
    if (misaligned(lse, 4) || misaligned(scores)) return MOE_ERR_ALIGN;
    a.q = q;
    a.lse = lse;
    a.scores = scores;
    a.ldq = ldq;
    a.Hq = g.heads;
    a.G = g.heads / g.kv_heads;
    a.causal = opt->causal;
    a.window = opt->window;
    a.scale2 = scale2_of(g);
    a.decay = opt->decay;
    a.part = ctx->part;
    a.tickets = ctx->tickets;
    return with_counters(ctx->tickets_clear, stream, [&](bool& clear, hipStream_t s) { return launch_kv_weights(g.dtype, g.kv_format == MOE_KV_FP8, a, clear, s); });
}

moe_status moe_kv_select(moe_kv_ctx* ctx, const float* scores, int64_t n_pages, const moe_kv_batch* batch, const moe_select_options* opt,
                         int32_t* keep, int32_t* keep_lens, void* stream)
{
    if (!ctx || !opt) return MOE_ERR_NULL;
    SelectArgs a;
    const moe_status st = view_of_tokens(ctx, n_pages, batch, &a.c);
    if (st != MOE_OK) return st;
    if (opt->budget < 1 || opt->budget > 1 << 30 || opt->first < 0 || opt->recent < 0 || opt->first > opt->budget - opt->recent) return MOE_ERR_SHAPE;
    if (a.c.S == 0) return MOE_OK;
    if (!scores || !keep || !keep_lens) return MOE_ERR_NULL;
    if (misaligned(scores) || misaligned(keep) || misaligned(keep_lens, 4)) return MOE_ERR_ALIGN;
    a.scores = scores;
    a.keep = keep;
    a.keep_lens = keep_lens;
    a.budget = opt->budget;
    a.first = opt->first;
    a.recent = opt->recent;
    return dev(launch_kv_select(a, ctx->part, part_bytes(ctx->cfg), static_cast<hipStream_t>(stream)));
}

moe_status moe_kv_compact(moe_kv_ctx* ctx, const moe_kv_pages* pages, const moe_kv_batch* batch, const moe_kv_keep* keep, float* scores, void* stream)
{
    if (!ctx || !pages || !keep) return MOE_ERR_NULL;
    CompactArgs a;
    const moe_status st = view_of_tokens(ctx, pages->n_pages, batch, &a.c);
    if (st != MOE_OK) return st;
    if (keep->max_keep < 0 || keep->max_keep > 1 << 30 || (keep->per_head != 0 && keep->per_head != 1)) return MOE_ERR_SHAPE;
    if (a.c.S == 0 || keep->max_keep == 0 || a.c.max_pages == 0) return MOE_OK;
    const moe_kv_config& g = ctx->cfg;
    const bool fp8 = g.kv_format == MOE_KV_FP8;
    if (!pages->k_pages || !pages->v_pages || (fp8 && (!pages->k_scales || !pages->v_scales)) || !keep->tokens || !keep->lens) return MOE_ERR_NULL;
    if (misaligned(pages->k_pages) || misaligned(pages->v_pages) || (fp8 && (misaligned(pages->k_scales) || misaligned(pages->v_scales))) ||
        misaligned(scores) || misaligned(keep->tokens, 4) || misaligned(keep->lens, 4) || misaligned(keep->first, 4))
        return MOE_ERR_ALIGN;
    a.c.k = static_cast<char*>(pages->k_pages);
    a.c.v = static_cast<char*>(pages->v_pages);
    a.c.ks = fp8 ? pages->k_scales : nullptr;
    a.c.vs = fp8 ? pages->v_scales : nullptr;
    a.scores = scores;
    a.tokens = keep->tokens;
    a.lens = keep->lens;
    a.first = keep->first;
    a.max_keep = keep->max_keep;
    a.per_head = keep->per_head;
    return with_counters(ctx->compact_clear, stream, [&](bool clear, hipStream_t s) {
        return launch_kv_compact(g.dim * (fp8 ? 1 : g.dtype == MOE_BF16 ? 2 : 4), a, ctx->compact_state, clear, s);
    });
}

}  // extern "C"
