// Shared by the kernels of the paged key/value cache (kv_cache.hip) and its attention (attention.hip).
#pragma once
#include "common.h"

namespace moe {

// A layer's pages and a batch's descriptors as the kernels take them.  Everything that comes from the descriptors is clamped or
// tested on the device before it becomes an address.
struct KVView {
    char *k, *v;
    uint8_t *ks, *vs;              // NULL unless the pages hold FP8 codes
    const int32_t *off, *lens, *table;
    int n_pages, S, max_pages;
    int T, Hk, D, page_shift;
};

// The 64-bit index of a token's row among the rows of all pages, [n_pages, Hk, page].
__device__ __forceinline__ int64_t page_row(int id, int Hk, int h, int shift, int slot)
{
    return ((((int64_t)id * Hk) + h) << shift) + slot;
}

// The factor that a scale byte stands for.
__device__ __forceinline__ float scale_of(uint32_t byte)
{
    const float f = __builtin_amdgcn_ldexpf(1.0f, (int)byte - 127);
    return byte == 255u ? __builtin_nanf("") : f;
}

// A launch has fewer than 2^32 threads, in blocks of 256 here.  What takes more is not launched: hipErrorInvalidConfiguration.
constexpr int64_t kMaxBlocks = ((int64_t)1 << 24) - 1;

// kv_cache.hip
hipError_t launch_kv_append(int dtype, bool fp8, const KVView& c, const void* k, int64_t ldk, const void* v, int64_t ldv, hipStream_t s);
hipError_t launch_kv_gather(int dtype, bool fp8, const KVView& c, void* k, int64_t ldk, void* v, int64_t ldv, hipStream_t s);

// attention.hip
struct AttnArgs {
    KVView c;
    const void* q;
    void* out;
    float* lse;
    const float* sinks;
    int64_t ldq, ldo;
    int Hq, G, causal, window;
    int few_rows, tile_rows;       // packed rows of a tile, up to few_rows and where a sequence has more (set by the launch, as are:)
    int tile_tokens;               // tile_rows / G
    int tile_items;                // items that a batch with tiles of many rows is cut into
    uint32_t g_magic, hk_magic;    // for divisions by G and by Hk
    float scale2;                  // log2(e) / sqrt(dim): scores are kept as powers of two
    float* part;                   // partial outputs, kPartUnits of 16 rows x D
    float2* part_stats;            // and their rows' maximum and sum
    uint32_t* tickets;             // kPartUnits, zero between launches
};
// Partial results are stored in units of 16 rows.
constexpr int kPartUnits = 8192;
// clear_tickets: they are not known to be zero
hipError_t launch_attention(int dtype, bool fp8, const AttnArgs& a, bool clear_tickets, hipStream_t s);

}  // namespace moe
