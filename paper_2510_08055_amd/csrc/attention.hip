// Attention of a batch's new rows to a paged key/value cache.
//
// For a row q of a head, over the tokens j it sees:  x_j = (q . k_j) log2(e) / sqrt(dim),  out = sum_j 2^(x_j - M) v_j / sum_j 2^(x_j - M),
// in one pass over the tokens with a running M and sum (a later maximum scales what has been summed so far).  The rows of all
// query heads that read one key/value head are one matrix: packed row r of a sequence is new token r / G, query head h G + r % G.
//
// Work is cut on the device, from the descriptors: every block of a launch reads them and finds its own item (sequence, key/value
// head, tile of packed rows, piece of the history), so no host ever waits for a length.  Pieces are as long as spreads the batch's work over
// the chip; a tile whose history is in several pieces is joined, from fp32 partial results, by the block that ends its last piece.
#include "attention_few.h"
#include "attention_tile.h"

namespace moe {
namespace {

template <typename T, bool FP8, int DP> constexpr int few_rows() { return DP <= 128 ? 32 : 16; }      // 32 rows of 256 dimensions do not fit the registers
template <typename T, bool FP8, int DP> constexpr size_t lds_bytes()
{
    const size_t few = sizeof(typename Few<T, FP8, DP, few_rows<T, FP8, DP>() / 16>::Shared);
    const size_t many = sizeof(T) == 2 ? Many<FP8, DP>::LDS : 0;
    return ((few > many ? few : many) + 15) / 16 * 16;
}

template <typename T, bool FP8, int DP> __global__ __launch_bounds__(256, sizeof(T) == 4 || DP > 128 ? 1 : 2) void attention_kernel(AttnArgs a)
{
    extern __shared__ __attribute__((aligned(256))) char smem[];
    constexpr int NQ = few_rows<T, FP8, DP>() / 16;
    const Item it = find_item(a, blockIdx.x, *reinterpret_cast<PlanShared*>(smem + lds_bytes<T, FP8, DP>()));
    if (!it.valid) return;
    if (it.q.many) {
        if constexpr (sizeof(T) == 2) Many<FP8, DP>::run(a, it, smem);
    } else if (it.q.units == 1) {
        Few<T, FP8, DP, 1>::run(a, it, *reinterpret_cast<typename Few<T, FP8, DP, 1>::Shared*>(smem));
    } else if constexpr (NQ > 1) {
        Few<T, FP8, DP, NQ>::run(a, it, *reinterpret_cast<typename Few<T, FP8, DP, NQ>::Shared*>(smem));
    }
}

template <typename T, bool FP8, int DP> hipError_t launch(AttnArgs a, hipStream_t s)
{
    a.few_rows = few_rows<T, FP8, DP>();
    a.tile_rows = sizeof(T) == 2 ? kManyRows : a.few_rows;
    a.tile_tokens = a.tile_rows / a.G;
    a.g_magic = map_magic_of(a.G);
    // a block for every item there can be: a tile for a sequence and for tile_rows more packed rows; pieces are kFewItems and kTileItems
    // more at most (and a few for the rounding of their lengths), fewer where no history is long
    const int64_t tiles = (int64_t)(a.c.S < a.c.T ? a.c.S : a.c.T) + (int64_t)a.c.T * a.G / a.tile_rows;
    const int64_t base = tiles * a.c.Hk;
    const int64_t longest = (int64_t)a.c.max_pages << a.c.page_shift;
    const int64_t by_length = longest > kMinPiece ? base * ((longest - 1) / kMinPiece) : 0;
    const int64_t most = kFewItems + kTileItems + 64;
    const int64_t grid = base + (by_length < most ? by_length : most) + 16;      // (either kind's items are dealt out by eights)
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    constexpr size_t lds = lds_bytes<T, FP8, DP>() + sizeof(PlanShared);
    static bool done[kMaxDevices];
    const auto kern = attention_kernel<T, FP8, DP>;
    const hipError_t e = ensure_lds_limit(kern, lds, done);
    if (e != hipSuccess) return e;
    kern<<<(unsigned)grid, 256, lds, s>>>(a);
    return hipGetLastError();
}

template <typename T, bool FP8> hipError_t launch_by_dim(const AttnArgs& a, hipStream_t s)
{
    if (a.c.D <= 64) return launch<T, FP8, 64>(a, s);
    if (a.c.D <= 128) return launch<T, FP8, 128>(a, s);
    return launch<T, FP8, 256>(a, s);
}

}  // namespace

hipError_t launch_attention(int dtype, bool fp8, const AttnArgs& a, hipStream_t s)
{
    if (dtype == MOE_BF16) return fp8 ? launch_by_dim<bf16_t, true>(a, s) : launch_by_dim<bf16_t, false>(a, s);
    return fp8 ? launch_by_dim<float, true>(a, s) : launch_by_dim<float, false>(a, s);
}

}  // namespace moe
