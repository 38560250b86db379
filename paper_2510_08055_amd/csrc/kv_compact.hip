// Moving the kept tokens of a sequence and head together, in place.
//
// Lists ascend, so a token moves to a lower slot or stays, and what a tile of tokens overwrites is read by this tile or by ones before it.  A block
// therefore reads its whole tile (keys, values, scale bytes, scores) into registers, says so, waits until the tiles before it have been read, and writes.
// Blocks draw their tiles in order: the tiles that one waits for were drawn before it, by blocks that are running and read without waiting for anything, so every
// wait ends.  What bounds it: memory, read and written once (16 histories of 8192 tokens in 8 heads halved, 541 MB, 116 us, 4.7 TB/s: a copy's rate; a block to a
// sequence and head, tile after tile, took 394; 256 such histories, 2048 lists, have more tiles than there are words of state and go that way: 1819 us,
// the same rate); for short lists a chain of loads (list, page table, rows) behind a launch, 3.5 us.
#include "kv.h"

namespace moe {
namespace {

// 16 bytes that nobody asks for again soon (16 histories: 122 us with plain stores, 116 so).
__device__ __forceinline__ void store_stream(void* p, uint4 v)
{
    typedef uint32_t uint32x4_t __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(__builtin_bit_cast(uint32x4_t, v), static_cast<uint32x4_t*>(p));
}

// A tile of a list: 256 / L tokens at a time, L lanes to a row of 16-byte pieces, U times.
template <int L, int U> struct Tile {
    static constexpr int PER = 256 / L, TOKENS = PER * U;
    uint4 k[U], v[U];
    uint32_t ks[U], vs[U];
    float w[U];
    int64_t from[U], to[U];        // rows of the pages; to: -1 where nothing moves

    // Where the tokens are and go (every load of a kind in flight together); whether one of this thread's moves.
    __device__ __forceinline__ bool find(const CompactArgs& a, int s, int h, int64_t i0, int64_t count)
    {
        const KVView& c = a.c;
        const int64_t first = a.first ? a.first[s] : 0;
        const int32_t* list = a.tokens + (a.per_head ? (int64_t)s * c.Hk + h : (int64_t)s) * a.max_keep;
        const int32_t* table = c.table + (int64_t)s * c.max_pages;
        const int mine = threadIdx.x / L, last = c.max_pages - 1;
        int token[U], id[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + u * PER + mine;
            token[u] = list[i < count ? i : count - 1];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t slot = first + i0 + u * PER + mine;
            const int64_t p[2] = {(int64_t)(token[u] >> c.page_shift), slot >> c.page_shift};
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const bool in = p[e] >= 0 && p[e] <= last;
                const int at = table[in ? p[e] : 0];
                id[u][e] = in ? at : -1;
            }
        }
        bool moves = false;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + u * PER + mine, slot = first + i;
            auto there = [&](int v) { return v >= 0 && v < c.n_pages; };
            const bool go = i < count && token[u] != slot && there(id[u][0]) && there(id[u][1]);
            const int mask = (1 << c.page_shift) - 1;
            from[u] = go ? page_row(id[u][0], c.Hk, h, c.page_shift, token[u] & mask) : 0;
            to[u] = go ? page_row(id[u][1], c.Hk, h, c.page_shift, (int)slot & mask) : -1;
            moves |= go;
        }
        return moves;
    }
    // (what does not move reads the first row of all, which is there)
    __device__ __forceinline__ void read(const CompactArgs& a, int row)
    {
        const KVView& c = a.c;
        const int at = threadIdx.x % L * 16 < row ? threadIdx.x % L * 16 : 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            k[u] = *reinterpret_cast<const uint4*>(c.k + from[u] * row + at);
            v[u] = *reinterpret_cast<const uint4*>(c.v + from[u] * row + at);
        }
        if (c.ks) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                ks[u] = c.ks[from[u]];
                vs[u] = c.vs[from[u]];
            }
        }
        if (a.scores) {
#pragma unroll
            for (int u = 0; u < U; ++u) w[u] = a.scores[from[u]];
        }
    }
    __device__ __forceinline__ void write(const CompactArgs& a, int row) const
    {
        const KVView& c = a.c;
        const int piece = threadIdx.x % L;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (to[u] < 0) continue;
            if (piece * 16 < row) {
                store_stream(c.k + to[u] * row + piece * 16, k[u]);
                store_stream(c.v + to[u] * row + piece * 16, v[u]);
            }
            if (piece == 0 && c.ks) {
                c.ks[to[u]] = (uint8_t)ks[u];
                c.vs[to[u]] = (uint8_t)vs[u];
            }
            if (piece == 0 && a.scores) a.scores[to[u]] = w[u];
        }
    }
};

__device__ __forceinline__ int64_t count_of(const CompactArgs& a, int s) { return a.lens[s] < a.max_keep ? a.lens[s] : a.max_keep; }

// Every thread's loads have arrived (what they read may be overwritten), and its stores.
__device__ __forceinline__ void all_arrived()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// A block to a sequence and head, tile after tile.
template <int L, int U> __global__ __launch_bounds__(256) void compact_kernel(CompactArgs a, int row)
{
    const int s = blockIdx.x / a.c.Hk, h = blockIdx.x - s * a.c.Hk;
    const int64_t count = count_of(a, s);
    for (int64_t i = 0; i < count; i += Tile<L, U>::TOKENS) {
        Tile<L, U> t;
        if (!__syncthreads_or(t.find(a, s, h, i, count))) continue;
        t.read(a, row);
        all_arrived();
        t.write(a, row);
    }
}

// A block to a tile.  state, of each sequence and head: the next tile to draw, the blocks that have ended, then a word for every tile that has
// been read; zero between launches: the block that ends last leaves it so.  A block counts itself as ended once its mark has arrived, so that no mark lands on a word
// that is cleared already (stores and atomics to different words keep no order of their own).  (One pair of counters for all blocks cost 16 histories 60 us of
// waiting for them.)
template <int L, int U> __global__ __launch_bounds__(256) void compact_tiles_kernel(CompactArgs a, int row, int items, int tiles, uint32_t* state)
{
    __shared__ uint32_t drawn;
    const int item = (int)(blockIdx.x % (uint32_t)items), s = item / a.c.Hk, h = item - s * a.c.Hk;
    uint32_t* const mine = state + (int64_t)item * (tiles + 2);
    if (threadIdx.x == 0) drawn = __hip_atomic_fetch_add(mine, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int64_t count = count_of(a, s);
    __syncthreads();
    const int tile = __builtin_amdgcn_readfirstlane((int)drawn);
    const int64_t i0 = (int64_t)tile * Tile<L, U>::TOKENS;
    if (i0 < count) {
        uint32_t* const read = mine + 2;
        Tile<L, U> t;
        const bool moves = __syncthreads_or(t.find(a, s, h, i0, count)) != 0;
        if (moves) t.read(a, row);
        all_arrived();
        if (threadIdx.x == 0) store_shared(read + tile, 1u);
        if (moves) {
            for (int i = threadIdx.x; i < tile; i += 256)
                while (load_shared(read + i) == 0) __builtin_amdgcn_s_sleep(2);
            __syncthreads();
            t.write(a, row);
        }
    }
    all_arrived();
    if (threadIdx.x == 0) drawn = __hip_atomic_fetch_add(mine + 1, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (drawn != (uint32_t)tiles - 1) return;
    for (int i = threadIdx.x; i < tiles + 2; i += 256) store_shared(mine + i, 0u);
}

template <int L> hipError_t launch(const CompactArgs& a, int row, int64_t items, uint32_t* state, hipStream_t s)
{
    // (8 times: 16 histories in tiles of 32 / 64 / 128 / 256 tokens, with one pair of counters, 412 / 239 / 181 / -, with a pair each - / 117 / 116 / 118)
    constexpr int U = 8, TOKENS = Tile<L, U>::TOKENS;
    const int64_t tiles = (a.max_keep + TOKENS - 1) / TOKENS;
    if (a.max_keep <= 256 / L) compact_kernel<L, 1><<<(unsigned)items, 256, 0, s>>>(a, row);
    else if (tiles == 1 || items * (tiles + 2) > kCompactWords) compact_kernel<L, U><<<(unsigned)items, 256, 0, s>>>(a, row);
    else compact_tiles_kernel<L, U><<<(unsigned)(items * tiles), 256, 0, s>>>(a, row, (int)items, (int)tiles, state);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_compact(int row, const CompactArgs& a, uint32_t* state, bool clear, hipStream_t s)
{
    const int64_t items = (int64_t)a.c.S * a.c.Hk;
    if (items > kMaxBlocks) return hipErrorInvalidConfiguration;
    if (clear) {
        const hipError_t e = launch_fill_zero(state, kCompactWords, s);
        if (e != hipSuccess) return e;
    }
    const int pieces = row / 16;
    if (pieces <= 4) return launch<4>(a, row, items, state, s);
    if (pieces <= 8) return launch<8>(a, row, items, state, s);
    if (pieces <= 16) return launch<16>(a, row, items, state, s);
    if (pieces <= 32) return launch<32>(a, row, items, state, s);
    return launch<64>(a, row, items, state, s);
}

}  // namespace moe
