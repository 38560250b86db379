// Attention of a batch's new rows to a paged key/value cache.
//
// For a row q of a head, over the tokens j it sees:  x_j = (q . k_j) log2(e) / sqrt(dim),  out = sum_j 2^(x_j - M) v_j / sum_j 2^(x_j - M),
// in one pass over the tokens with a running M and sum (a later maximum scales what has been summed so far).  The rows of all
// query heads that read one key/value head are one matrix: packed row r of a sequence is new token r / G, query head h G + r % G.
//
// Work is cut on the device, from the descriptors: every block of a launch reads them and finds its own item (sequence, key/value
// head, tile of packed rows, piece of the history), so no host ever waits for a length.  Pieces are as long as spreads the batch's work over
// the chip; a tile whose history is in several pieces is joined, from fp32 partial results, by the block that ends its last piece.
#pragma once
#include "attention_few.h"
#include "attention_tile.h"

namespace moe {
namespace {

// The kernel of a batch.  LIGHT: every tile has 16 rows, which needs fewer registers, so that more blocks share a unit.
template <typename T, bool FP8, int DP, bool EXACT, bool LIGHT, bool TREE> struct Kernel {
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int NQ = LIGHT || DP > 128 ? 1 : 2;      // (32 rows of 256 dimensions do not fit the registers)
    static constexpr bool MANY = !F32 && !LIGHT;
    static constexpr int BLOCKS = LIGHT ? (F32 ? (DP > 128 ? 1 : 2) : DP > 128 ? (FP8 ? 2 : 1) : DP > 64 ? (FP8 || EXACT ? 3 : 2) : 4) : (F32 || DP > 128 ? 1 : 2);      // of a unit
    static constexpr size_t PLAN_AT = ((MANY && Many<FP8, DP, EXACT, TREE>::LDS > sizeof(typename Few<T, FP8, DP, NQ, EXACT, TREE>::Shared) ? Many<FP8, DP, EXACT, TREE>::LDS
                                                                                                             : sizeof(typename Few<T, FP8, DP, NQ, EXACT, TREE>::Shared)) + 15) / 16 * 16;
    static constexpr size_t LDS = PLAN_AT + sizeof(PlanShared);
};

template <typename T, bool FP8, int DP, bool EXACT, bool LIGHT, bool TREE> __global__ __launch_bounds__(256, (Kernel<T, FP8, DP, EXACT, LIGHT, TREE>::BLOCKS)) void attention_kernel(AttnArgs a)
{
    typedef Kernel<T, FP8, DP, EXACT, LIGHT, TREE> K;
    extern __shared__ __attribute__((aligned(256))) char smem[];
    const Item it = find_item<TREE>(a, blockIdx.x, *reinterpret_cast<PlanShared*>(smem + K::PLAN_AT));
    if (!it.valid) return;
    if constexpr (K::MANY) {
        if (it.q.many) {
            Many<FP8, DP, EXACT, TREE>::run(a, it, smem);
            return;
        }
    }
    if constexpr (K::NQ > 1) {
        if (it.q.units > 1) {
            Few<T, FP8, DP, K::NQ, EXACT, TREE>::run(a, it, *reinterpret_cast<typename Few<T, FP8, DP, K::NQ, EXACT, TREE>::Shared*>(smem));
            return;
        }
    }
    Few<T, FP8, DP, 1, EXACT, TREE>::run(a, it, *reinterpret_cast<typename Few<T, FP8, DP, 1, EXACT, TREE>::Shared*>(smem));
}

template <typename T, bool FP8, int DP, bool EXACT, bool LIGHT, bool TREE> hipError_t launch(AttnArgs a, bool clear_tickets, hipStream_t s)
{
    typedef Kernel<T, FP8, DP, EXACT, LIGHT, TREE> K;
    a.few_rows = K::NQ * 16;
    a.tile_rows = K::MANY ? kManyRows : a.few_rows;
    a.tile_tokens = a.tile_rows / a.G;
    // a block for every item there can be: a tile for a sequence and for tile_rows more packed rows
    const int64_t tiles = (int64_t)(a.c.S < a.c.T ? a.c.S : a.c.T) + (int64_t)a.c.T * a.G / a.tile_rows;
    const int64_t base = tiles * a.c.Hk;
    if (base > kMaxBlocks) return hipErrorInvalidConfiguration;
    int units = 0;
    hipError_t e = compute_units(&units);
    if (e != hipSuccess) return e;
    a.tile_items = units * K::BLOCKS;
    a.g_magic = map_magic_of(a.G);
    a.hk_magic = map_magic_of(a.c.Hk);
    // pieces are kFewItems and tile_items more at most (and a few for the rounding of their lengths), fewer where no history is long
    const int64_t longest = (int64_t)a.c.max_pages << a.c.page_shift;
    const int64_t by_length = longest > kMinPiece ? base * ((longest - 1) / kMinPiece) : 0;
    const int64_t most = kFewItems + a.tile_items + 64;
    const int64_t grid = base + (by_length < most ? by_length : most) + 16;      // (those of many rows are rounded up to eights)
    if (grid > kMaxBlocks) return hipErrorInvalidConfiguration;
    static bool done[kMaxDevices];
    const auto kern = attention_kernel<T, FP8, DP, EXACT, LIGHT, TREE>;
    e = ensure_lds_limit(kern, K::LDS, done);
    if (e != hipSuccess) return e;
    if (clear_tickets && (e = launch_fill_zero(a.tickets, kPartUnits, s)) != hipSuccess) return e;
    kern<<<(unsigned)grid, 256, K::LDS, s>>>(a);
    return hipGetLastError();
}

template <typename T, bool FP8, int DP, bool TREE> hipError_t launch_by_rows(const AttnArgs& a, bool clear, hipStream_t s)
{
    // How rows spread over the sequences only the device knows.  Either kernel is right for any spread; a batch is taken for one of decode rows
    // (or drafted ones) with no more than 16 packed rows to a sequence on average, and where no sequence can have more than a few tiles' worth
    // of them: all but one row of every other sequence, or, with fewer rows than sequences, where empty ones are certain, all rows.
    // Measured, us, kernel with many-row tiles / the light one.  Batches of decode or drafted rows: dim 128, 64 sequences of up to 7000 tokens, 8 key/value
    // heads 273 / 259, FP8 164 / 149, 4 of them 155 / 145, FP8 91 / 78; 16 of four drafted rows over up to 1500 tokens 23 / 20, FP8 19 / 15.  Beside
    // 256 decode rows, 32 heads over 8, a prompt over 7680 tokens of 16 rows 147 / 177, 64 rows 151 / 236, 128 rows 156 / 245, 200 rows 163 / 353, 512 rows 197 / 455.
    // fp32 batches have no tiles of many rows to lose: there the average alone decides (256 decode rows beside 512 prompt rows, us, tiles of 32 / of 16: dim 128,
    // 32 heads over 8 410 / 331, over 7680 tokens 1116 / 1122; dim 64, 32 over 32 641 / 532, 1005 / 943).
    constexpr int kMostRows = 3 * kManyRows;
    const int64_t rows = a.c.T, seqs = a.c.S, most = rows < seqs ? rows : rows - seqs + 1;
    const bool light = rows * a.G <= 16 * seqs && (sizeof(T) == 4 || most * a.G <= kMostRows);
    if constexpr (sizeof(T) == 2) {
        if (a.c.D == DP) return light ? launch<T, FP8, DP, true, true, TREE>(a, clear, s) : launch<T, FP8, DP, true, false, TREE>(a, clear, s);
    }
    return light ? launch<T, FP8, DP, false, true, TREE>(a, clear, s) : launch<T, FP8, DP, false, false, TREE>(a, clear, s);
}

template <typename T, bool FP8, bool TREE> hipError_t launch_by_dim(const AttnArgs& a, bool clear, hipStream_t s)
{
    if (a.c.D <= 64) return launch_by_rows<T, FP8, 64, TREE>(a, clear, s);
    if (a.c.D <= 128) return launch_by_rows<T, FP8, 128, TREE>(a, clear, s);
    return launch_by_rows<T, FP8, 256, TREE>(a, clear, s);
}

template <bool TREE> hipError_t launch_by_type(int dtype, bool fp8, const AttnArgs& a, bool clear, hipStream_t s)
{
    if (dtype == MOE_BF16) return fp8 ? launch_by_dim<bf16_t, true, TREE>(a, clear, s) : launch_by_dim<bf16_t, false, TREE>(a, clear, s);
    return fp8 ? launch_by_dim<float, true, TREE>(a, clear, s) : launch_by_dim<float, false, TREE>(a, clear, s);
}

}  // namespace
}  // namespace moe
