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
    const uint64_t* masks;         // of trees, [T, words]: bit j of row i: it sees row j of its sequence (words: 0 without trees)
    const int32_t* positions;      // of their rows, read with a window alone
    int words;
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
// tree_attention.hip: the same with masks
hipError_t launch_tree_attention(int dtype, bool fp8, const AttnArgs& a, bool clear_tickets, hipStream_t s);


// kv_tree.hip
constexpr int kMaxTreeWords = 16;      // of 64 rows each
hipError_t launch_tree_masks(const KVView& c, const int32_t* parents, int words, int window, uint64_t* masks, int32_t* positions, hipStream_t s);

// kv_weights.hip
struct WeightArgs {
    KVView c;
    const void* q;
    const float* lse;
    float* scores;
    int64_t ldq;
    int Hq, G, causal, window;
    uint32_t g_magic;              // (set by the launch, as is:)
    int few_rows;                  // packed rows of the sequences that the kernel of few rows takes
    int split_chunks;              // of 256 sequences, for whose partial sums there are slots
    float scale2, decay;
    float* part;                   // partial sums of tokens, and tickets, as in AttnArgs
    uint32_t* tickets;
};
// clear_tickets: as above; false again where the tickets were not needed, and so not cleared
hipError_t launch_kv_weights(int dtype, bool fp8, const WeightArgs& a, bool& clear_tickets, hipStream_t s);

// kv_select.hip
struct SelectArgs {
    KVView c;
    const float* scores;
    int32_t *keep, *keep_lens;
    int budget, first, recent;
};
hipError_t launch_kv_select(const SelectArgs& a, void* workspace, size_t bytes, hipStream_t s);      // (the workspace need not be clear)

// kv_compact.hip; row: bytes of a token's keys
struct CompactArgs {
    KVView c;
    float* scores;
    const int32_t *tokens, *lens, *first;
    int64_t max_keep;
    int per_head;
};
// words of state, zero between launches: how far the tiles of a launch are
constexpr int kCompactWords = 1 << 16;
hipError_t launch_kv_compact(int row, const CompactArgs& a, uint32_t* state, bool clear, hipStream_t s);

}  // namespace moe
