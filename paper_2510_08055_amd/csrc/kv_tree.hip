// Ancestor masks and positions of trees of drafted tokens, from their rows' parents.
//
// A thread takes a row of a tree.  What a row reaches by fewer than 2^k steps to its parent, and the row that 2^k steps lead to, follow from the same
// of that row: mask_{k+1}(i) = mask_k(i) | mask_k(up_k(i)), up_{k+1}(i) = up_k(up_k(i)), so the longest path of n rows takes log2(n) rounds.
// What bounds it is latency: ends of the sequences, parents, the rounds in LDS, the stores: 16 trees of 8 rows 3.0 us, 256 of 33 to 200 rows beside a prompt 5.3.
#include "kv.h"

namespace moe {
namespace {

// Words of a mask: W, a power of two, of which the tensor has `words`.  A block holds a tree; blockIdx.y shares the rows of prompts.
template <int W> __global__ __launch_bounds__(64 * W) void tree_masks_kernel(KVView c, const int32_t* __restrict__ parents, int words,
                                                                             int window, uint64_t* __restrict__ masks, int32_t* __restrict__ positions)
{
    extern __shared__ __attribute__((aligned(16))) uint64_t reach[];      // [word][row], then the rows' ups
    int32_t* ups = reinterpret_cast<int32_t*>(reach + W * 64 * W);
    const int s = blockIdx.x, i = threadIdx.x;
    const int lo = c.off[s], hi = c.off[s + 1], len = c.lens[s];
    if (lo < 0 || hi <= lo || hi > c.T) return;
    const int n = hi - lo, p0 = (len > 0 ? len : 0) - n;
    if (n > 64 * words) {
        for (int64_t r = (int64_t)blockIdx.y * (64 * W) + i; r < n; r += (int64_t)gridDim.y * (64 * W)) {
            for (int w = 0; w < words; ++w) masks[(lo + r) * words + w] = 0;
            if (positions) positions[lo + r] = p0 + (int)r;
        }
        return;
    }
    if (blockIdx.y > 0) return;
    int up = i < n ? parents[lo + i] : -1;
    up = up < i ? up : -1;                         // (parents come before their children, so no path comes back)
    uint64_t mine[W];
#pragma unroll
    for (int w = 0; w < W; ++w) mine[w] = i >> 6 == w ? 1ull << (i & 63) : 0;
    for (;;) {
#pragma unroll
        for (int w = 0; w < W; ++w) reach[w * 64 * W + i] = mine[w];
        ups[i] = up;
        if (!__syncthreads_or(up >= 0)) break;
        int next = -1;
        if (up >= 0) {
#pragma unroll
            for (int w = 0; w < W; ++w) mine[w] |= reach[w * 64 * W + up];
            next = ups[up];
        }
        up = next;
        __syncthreads();
    }
    if (i >= n) return;
    int count = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) count += __popcll(mine[w]);
    if (positions) positions[lo + i] = p0 + count - 1;
    // A window leaves the last ancestors, those of the highest rows: whole words go first.
    int drop = window > 0 && count > window ? count - window : 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const int here = __popcll(mine[w]);
        if (drop >= here) {
            if (drop > 0) mine[w] = 0;
            drop -= here;
        } else {
            for (; drop > 0; --drop) mine[w] &= mine[w] - 1;
        }
        if (w < words) masks[(int64_t)(lo + i) * words + w] = mine[w];
    }
}

template <int W> hipError_t launch(const KVView& c, const int32_t* parents, int words, int window, uint64_t* masks, int32_t* positions, hipStream_t s)
{
    static bool done[kMaxDevices];
    constexpr size_t lds = (size_t)W * 64 * W * 8 + 64 * W * 4;
    const hipError_t e = ensure_lds_limit(tree_masks_kernel<W>, lds, done);
    if (e != hipSuccess) return e;
    // blocks for the rows of prompts, if there can be any
    const int more = c.T <= 64 * words || c.S > 4096 ? 1 : c.T / 4096 < 31 ? c.T / 4096 + 1 : 32;
    tree_masks_kernel<W><<<dim3((unsigned)c.S, (unsigned)more), 64 * W, lds, s>>>(c, parents, words, window, masks, positions);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_masks(const KVView& c, const int32_t* parents, int words, int window, uint64_t* masks, int32_t* positions, hipStream_t s)
{
    if (words <= 1) return launch<1>(c, parents, words, window, masks, positions, s);
    if (words <= 2) return launch<2>(c, parents, words, window, masks, positions, s);
    if (words <= 4) return launch<4>(c, parents, words, window, masks, positions, s);
    if (words <= 8) return launch<8>(c, parents, words, window, masks, positions, s);
    return launch<16>(c, parents, words, window, masks, positions, s);
}

}  // namespace moe
