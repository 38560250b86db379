// Moving the kept tokens of a sequence and head together, in place.
//
// Lists ascend, so a token moves to a lower slot or stays: a block that takes a list from its front, reads a tile of tokens whole before it writes
// them, and goes on to the next, never writes a slot that is still to be read.
#include "kv.h"

namespace moe {
namespace {

// Index of a token's row among the rows of all pages, -1 where it is not there.
__device__ __forceinline__ int64_t place_of(const KVView& c, int s, int h, int64_t token)
{
    const int64_t p = token >> c.page_shift;
    if (token < 0 || p >= c.max_pages) return -1;
    const int id = c.table[(int64_t)s * c.max_pages + p];
    if (id < 0 || id >= c.n_pages) return -1;
    return page_row(id, c.Hk, h, c.page_shift, (int)token & ((1 << c.page_shift) - 1));
}

// A block: the keys (blockIdx.y 0) or the values (1) of a sequence and head.  L: lanes of a token, 16 bytes each.
constexpr int U = 4;
template <int L> __global__ __launch_bounds__(256) void compact_kernel(CompactArgs a, int row)
{
    const KVView& c = a.c;
    const int s = blockIdx.x / c.Hk, h = blockIdx.x - s * c.Hk, values = blockIdx.y;
    const int64_t count = a.lens[s] < a.max_keep ? a.lens[s] : a.max_keep;
    const int64_t first = a.first ? a.first[s] : 0;
    const int32_t* list = a.tokens + (a.per_head ? (int64_t)blockIdx.x : (int64_t)s) * a.max_keep;
    char* pages = values ? c.v : c.k;
    uint8_t* scales = values ? c.vs : c.ks;
    float* scores = values ? nullptr : a.scores;
    constexpr int PER = 256 / L;
    const int piece = threadIdx.x % L, mine = threadIdx.x / L;
    for (int64_t i0 = 0; i0 < count; i0 += PER * U) {
        uint4 x[U];
        uint8_t sc[U];
        float w[U];
        int64_t to[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + u * PER + mine;
            to[u] = -1;
            if (i >= count) continue;
            const int64_t from = place_of(c, s, h, list[i]);
            if (from < 0) continue;
            to[u] = place_of(c, s, h, first + i);
            if (to[u] == from) to[u] = -1;
            if (to[u] < 0) continue;
            if (piece * 16 < row) x[u] = *reinterpret_cast<const uint4*>(pages + from * row + piece * 16);
            if (piece == 0 && scales) sc[u] = scales[from];
            if (piece == 0 && scores) w[u] = scores[from];
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (to[u] < 0) continue;
            if (piece * 16 < row) *reinterpret_cast<uint4*>(pages + to[u] * row + piece * 16) = x[u];
            if (piece == 0 && scales) scales[to[u]] = sc[u];
            if (piece == 0 && scores) scores[to[u]] = w[u];
        }
    }
}

}  // namespace

hipError_t launch_kv_compact(int row, const CompactArgs& a, hipStream_t s)
{
    const int64_t blocks = (int64_t)a.c.S * a.c.Hk;
    if (2 * blocks > kMaxBlocks) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks, 2);
    const int pieces = row / 16;
    if (pieces <= 4) compact_kernel<4><<<grid, 256, 0, s>>>(a, row);
    else if (pieces <= 8) compact_kernel<8><<<grid, 256, 0, s>>>(a, row);
    else if (pieces <= 16) compact_kernel<16><<<grid, 256, 0, s>>>(a, row);
    else if (pieces <= 32) compact_kernel<32><<<grid, 256, 0, s>>>(a, row);
    else compact_kernel<64><<<grid, 256, 0, s>>>(a, row);
    return hipGetLastError();
}

}  // namespace moe
