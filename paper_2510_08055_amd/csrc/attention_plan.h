// What the attention's kernels share: the plan that finds a block's work, and how finished rows are stored.
#pragma once
#include <cfloat>

#include "kv.h"

namespace moe {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef float float16_t __attribute__((ext_vector_type(16)));

constexpr float kLowest = -FLT_MAX;      // a running maximum before its first token: finite, so that no difference is NaN
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// Items that the pieces of a launch aim at: of few rows, kFewItems, and with many rows among them, a round of the blocks that the
// units hold at once (AttnArgs::tile_items).  Pieces are multiples of kMinPiece tokens (a step of 32 for each of a block's four waves), and no
// shorter than kMinTilePiece where a tile has many rows: a piece more costs its partial results, 64 KB at dim 128.
// Measured, us, kFewItems 384 / 512 / 1024 / 2048: 128 ragged histories of up to 8192 tokens 152 / 139 / 136 / 139, 24 drafted ones over FP8 106 / 120 /
// 120 / 125 (how the last pieces fall), 32 of up to 4096 tokens 31 / 29 / 35 / 41, 128 of up to 1024 29 / 27 / 29 / 34.  (Equal stretches of all the
// work laid end to end, one to a block, bring the first two to 127 and 104, but their longer plan costs every launch 2 us, and the
// others 20 to 40 %.)
// kMinTilePiece 256 / 512 / 768: 300 prompt rows 19 / 17 / 17, 16 drafts of 9 rows over up to 6000 tokens 40 / 31 / 33.
constexpr int kFewItems = 512;
constexpr int kMinPiece = 128, kMinTilePiece = 512;

// TREE, here and below: the batch's short sequences are drafts whose rows see their ancestors (AttnArgs::masks) instead of all rows before them.
struct Seq {
    int row0, n, kv;                // first row, rows, tokens with them (of which the table need not reach all: held_of)
    int tiles, units, len;          // tiles of packed rows, units of 16 rows to a tile, tokens of the longest tile's range
    bool many;                      // its tiles are those of attention_tile.h
};
struct Item {
    Seq q;
    int seq, head, tile, sub;       // sub: the piece
    int piece;                      // tokens of a piece; 0: the history is in one
    int slot;                       // of the partial results: first unit of the tile's first piece
    bool valid;
};

// The tokens of a sequence that can be there, those its row of the table reaches.  Positions are taken from its length as it is.
__device__ __forceinline__ int held_of(const KVView& c, int kv)
{
    const int most = c.max_pages << c.page_shift;
    return kv < most ? kv : most;
}

template <bool TREE> __device__ __forceinline__ bool is_tree(const AttnArgs& a, int n) { return TREE && n <= 64 * a.words; }

template <bool TREE> __device__ __forceinline__ Seq shape_of(const AttnArgs& a, int lo, int hi, int kv)
{
    Seq q;
    q.row0 = lo;
    q.n = hi - lo;
    q.kv = kv < 0 ? 0 : kv;
    const int rows = q.n * a.G;
    q.many = rows > a.few_rows && a.tile_rows > a.few_rows;
    const int per = rows <= 16 ? 16 : rows <= a.few_rows ? a.few_rows : a.tile_rows;      // (all powers of two)
    q.units = per / 16;
    q.tiles = (rows + per - 1) >> (31 - __builtin_clz(per));
    q.len = held_of(a.c, q.kv);
    if (a.window > 0) {                                      // (windows, rows and what the table reaches are at most 2^30)
        const int first = q.kv - q.n - a.window + 1;
        int len = q.len - (first > 0 ? first : 0) + 31;
        const int one = a.window + a.tile_tokens + 2 + 31;
        if (a.causal && !is_tree<TREE>(a, q.n) && one < len) len = one;
        if (len < q.len) q.len = len > 0 ? len : 0;
    }
    return q;
}

__device__ __forceinline__ int last_lane(int v) { return __builtin_amdgcn_readlane(v, 63); }
__device__ __forceinline__ float last_lane(float v) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63)); }

// v / d for d > 1, from magic = ceil(2^32 / d), which overshoots by one at most.
__device__ __forceinline__ uint32_t divided(uint32_t v, uint32_t d, uint32_t magic)
{
    const uint32_t q = __umulhi(v, magic);
    return q * d > v ? q - 1 : q;
}

struct PlanShared {
    float work[2][4];
    int sums[3][4], bad[4];
    int found[9];
};

// The item of a block, the same in all of its threads.  A thread takes a sequence (256 at a time), so that the code is short: every
// block of a launch runs it before it can load anything, and code that runs once costs its instruction misses.  Up to 64 sequences
// every wave does it for itself, and nothing goes through LDS.
// Offsets that descend, or leave [0, T], would name rows twice or none: then there are no items at all.
template <bool TREE> __device__ __forceinline__ Item find_item(const AttnArgs& a, int block, PlanShared& sh)
{
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int S = a.c.S, Hk = a.c.Hk;
    const bool alone = S <= 64;
    const int me = alone ? lane : (int)threadIdx.x;
    Seq q;
    bool bad = false;
    auto load = [&](int b) {
        const int s = b + me;
        const int lo = a.c.off[s < S ? s : S], hi = a.c.off[s < S ? s + 1 : S], kv = a.c.lens[s < S ? s : S - 1];
        bad |= (lo < 0) | (hi < lo) | (hi > a.c.T);
        q = shape_of<TREE>(a, lo, bad ? lo : hi, kv);
    };
    // the batch's work in tokens of a tile, of few rows and of many
    float few = 0, many = 0;
    for (int b = 0; b < S; b += 256) {
        load(b);
        const float w = (float)q.tiles * (float)q.len;
        (q.many ? many : few) += w;
    }
    few = wave_scan(few);
    many = wave_scan(many);
    bool any_bad = __any(bad);
    Item it;
    it.valid = false;
    if (alone) {
        few = last_lane(few);
        many = last_lane(many);
    } else {
        if (lane == 63) {
            sh.work[0][wave] = few;
            sh.work[1][wave] = many;
            sh.bad[wave] = any_bad;
        }
        __syncthreads();
        any_bad = (sh.bad[0] | sh.bad[1] | sh.bad[2] | sh.bad[3]) != 0;
        few = sh.work[0][0] + sh.work[0][1] + sh.work[0][2] + sh.work[0][3];
        many = sh.work[1][0] + sh.work[1][1] + sh.work[1][2] + sh.work[1][3];
    }
    if (any_bad) return it;
    few *= (float)Hk;
    many *= (float)Hk;
    // A token costs an item of either kind about the same time (of a unit's share of the memory, or of its matrix cores).
    auto even = [](float work, int items, int least) {
        const float v = work * (1.0f / (float)items);
        return v <= (float)least ? least : v < 1e9f ? ((int)v + kMinPiece) / kMinPiece * kMinPiece : 1 << 30;
    };
    int few_piece = even(few, kFewItems, kMinPiece), many_piece = even(few + many, a.tile_items, kMinTilePiece);

    // items of many rows and of few, and units of partial results, of this thread's sequence
    int count[2], need, pieces;
    auto count_items = [&]() {
        const int piece = q.many ? many_piece : few_piece;
        pieces = q.len > piece ? (q.len + piece - 1) / piece : 1;
        const int n = q.tiles * Hk * pieces;
        count[0] = q.many ? n : 0;
        count[1] = q.many ? 0 : n;
        need = pieces > 1 ? n * q.units : 0;
    };
    int total[3] = {0, 0, 0}, incl[3], below[3] = {0, 0, 0};
    // inclusive sums over the sequences so far: incl (of the wave) + below (of the waves before)
    auto scan = [&](int c0, int c1, int c2) {
        incl[0] = wave_scan(c0);
        incl[1] = wave_scan(c1);
        incl[2] = wave_scan(c2);
        if (alone) {
#pragma unroll
            for (int k = 0; k < 3; ++k) total[k] = last_lane(incl[k]);
            return;
        }
        __syncthreads();
        if (lane == 63) {
#pragma unroll
            for (int k = 0; k < 3; ++k) sh.sums[k][wave] = incl[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            below[k] = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int v = sh.sums[k][w];
                below[k] += w < wave ? v : 0;
                total[k] += v;
            }
        }
    };
    for (;;) {
        int c0 = 0, c1 = 0, c2 = 0;
        for (int b = 0; b < S; b += 256) {
            if (S > 256) load(b);
            count_items();
            c0 += count[0];
            c1 += count[1];
            c2 += need;
        }
        total[0] = total[1] = total[2] = 0;
        scan(c0, c1, c2);
        if (total[2] <= kPartUnits) break;
        few_piece = many_piece = 1 << 30;      // (more pieces than the workspace holds: none are split)
    }
    // Tiles of many rows come first: they take longest.  (As many blocks as eights of them, so that an item's number still decides its
    // XCD.  512 prompt rows over 7680 tokens beside 32 decode rows, us: this order 117, decode rows first 121, both in turn 139.)
    const int first = (total[0] + 7) / 8 * 8, kind = block < first ? 0 : 1;
    if (kind == 1) block -= first;
    if (block >= total[kind]) return it;
    int rem = 0, pc = 1;
    auto found = [&](int b, int slots, auto put) {
        const int n = count[kind], r = block - (below[kind] + incl[kind] - n);
        const bool here = r >= 0 && r < n;
        put(here, q.row0, q.n, q.kv, q.tiles, q.units, b + me, r, pieces, slots + below[2] + incl[2] - need);
    };
    if (alone) {
        found(0, 0, [&](bool here, int row0, int n, int kv, int tiles, int units, int seq, int r, int p, int slot) {
            const int src = __ffsll((long long)__ballot(here)) - 1;
            auto get = [&](int v) { return __builtin_amdgcn_readlane(v, src); };
            it.q.row0 = get(row0); it.q.n = get(n); it.q.kv = get(kv); it.q.tiles = get(tiles); it.q.units = get(units);
            it.seq = get(seq); rem = get(r); pc = get(p); it.slot = get(slot);
        });
    } else {
        if (S > 256) total[0] = total[1] = total[2] = 0;
        for (int b = 0; b < S; b += 256) {
            int slots = 0;
            if (S > 256) {
                const int before = total[kind];
                slots = total[2];
                load(b);
                count_items();
                scan(count[0], count[1], need);
                below[kind] += before;
            }
            found(b, slots, [&](bool here, int row0, int n, int kv, int tiles, int units, int seq, int r, int p, int slot) {
                if (here) {
                    sh.found[0] = row0; sh.found[1] = n; sh.found[2] = kv; sh.found[3] = tiles; sh.found[4] = units;
                    sh.found[5] = seq; sh.found[6] = r; sh.found[7] = p; sh.found[8] = slot;
                }
            });
            if (S > 256 && block < total[kind]) break;
        }
        __syncthreads();
        auto get = [&](int i) { return __builtin_amdgcn_readfirstlane(sh.found[i]); };
        it.q.row0 = get(0); it.q.n = get(1); it.q.kv = get(2); it.q.tiles = get(3); it.q.units = get(4);
        it.seq = get(5); rem = get(6); pc = get(7); it.slot = get(8);
    }
    it.q.many = kind == 0;
    // Heads side by side, then tiles, long ones first, then pieces.  (Consecutive blocks go to the XCDs in turn: a head's tiles meet on
    // few of them, and no XCD is left with the last pieces, which short tiles do not have.)
    const int across = Hk == 1 ? rem : (int)divided((uint32_t)rem, (uint32_t)Hk, a.hk_magic);
    it.head = rem - across * Hk;
    it.sub = pc == 1 ? 0 : across / it.q.tiles;
    it.tile = it.q.tiles - 1 - (across - it.sub * it.q.tiles);
    it.piece = pc == 1 ? 0 : it.q.many ? many_piece : few_piece;
    it.slot += (it.tile * Hk + it.head) * pc * it.q.units;
    it.valid = true;
    return it;
}

// The new token of packed row r: r / G.
__device__ __forceinline__ int token_of(const AttnArgs& a, int r)
{
    return a.G == 1 ? r : (int)divided((uint32_t)r, (uint32_t)a.G, a.g_magic);
}

// The tokens that a tile's rows see: all rows those of [full_lo, full_hi), some row those of [lo, hi); lo is a multiple of 32.
struct Range {
    int p0;                         // position of the sequence's first row
    int held;                       // tokens of the sequence that can be there
    int rows, first;                // packed rows of the sequence, the tile's first
    int lo, hi, full_lo, full_hi;
    int pieces;
    int begin, end;                 // tokens of the item's piece
};
template <bool TREE> __device__ __forceinline__ Range range_of(const AttnArgs& a, const Item& it)
{
    Range r;
    const bool tree = is_tree<TREE>(a, it.q.n);
    r.rows = it.q.n * a.G;
    r.first = it.tile * it.q.units * 16;
    const int end = r.first + it.q.units * 16;
    const int last = (end < r.rows ? end : r.rows) - 1;
    r.p0 = it.q.kv - it.q.n;
    r.held = held_of(a.c, it.q.kv);
    // (a tree's rows stand anywhere from its root's position to its last row's, and all of them see what is cached before it)
    const int p_first = tree ? r.p0 : r.p0 + token_of(a, r.first), p_last = tree ? it.q.kv - 1 : r.p0 + token_of(a, last);
    r.hi = a.causal && p_last + 1 < r.held ? p_last + 1 : r.held;
    if (r.hi < 0) r.hi = 0;
    const int all_see = tree ? r.p0 : p_first + 1;
    r.full_hi = a.causal && all_see < r.held ? all_see : r.held;
    r.lo = a.window > 0 && p_first - a.window + 1 > 0 ? p_first - a.window + 1 : 0;
    r.full_lo = a.window > 0 && p_last - a.window + 1 > 0 ? p_last - a.window + 1 : 0;
    r.lo &= ~31;
    const int len = r.hi > r.lo ? r.hi - r.lo : 0;
    r.pieces = it.piece > 0 && len > it.piece ? (len + it.piece - 1) / it.piece : 1;
    r.begin = r.lo;
    r.end = r.hi;
    if (r.pieces > 1) {
        // (nearly) equal pieces, whole steps of every kernel
        const int steps = (len + kMinPiece - 1) / kMinPiece, each = steps / r.pieces, extra = steps - each * r.pieces;
        r.begin += (it.sub * each + (it.sub < extra ? it.sub : extra)) * kMinPiece;
        const int end = r.begin + (each + (it.sub < extra ? 1 : 0)) * kMinPiece;
        if (end < r.end) r.end = end;
    }
    return r;
}

// The first c of 64 bits.
__device__ __forceinline__ uint64_t first_bits(int c) { return c <= 0 ? 0 : c >= 64 ? ~0ull : (1ull << c) - 1; }

// The tokens that a row sees.
template <bool TREE> struct Sight {
    int lo, hi;                     // tokens [lo, hi)
    __device__ __forceinline__ void step(const AttnArgs&, int) {}
    __device__ __forceinline__ bool sees(int tok) const { return (tok < hi) & (tok >= lo); }
};
template <> struct Sight<true> {
    int lo, hi;                     // tokens [lo, hi), and where `row` is not negative,
    int row, p0, held;              // tokens p0 + j, before `held`, for the bits j of the row's mask
    int t;
    uint64_t bits;                  // bit i: token t + i
    // Every row of a wave before the tokens t .. t + 63 are asked for: two words of the mask hold them.
    __device__ __forceinline__ void step(const AttnArgs& a, int tok)
    {
        t = tok;
        bits = first_bits(hi - t) & ~first_bits(lo - t);
        const int at = t - p0;
        if (row >= 0 && at > -64 && at < 64 * a.words) {
            const uint64_t* m = a.masks + (int64_t)row * a.words;
            uint64_t w;
            if (at < 0) {
                w = m[0] << -at;
            } else {
                const int i = at >> 6, r = at & 63;
                w = m[i] >> r;
                if (r > 0 && i + 1 < a.words) w |= m[i + 1] << (64 - r);
            }
            bits |= w & first_bits(held - t);
        }
    }
    __device__ __forceinline__ bool sees(int tok) const { return ((bits >> (tok - t)) & 1) != 0; }
};

// What a packed row sees and where it lives.
template <bool TREE> struct Row {
    bool there;
    int row, head;                  // of the batch, of the queries
    Sight<TREE> sight;
};
template <bool TREE> __device__ __forceinline__ Row<TREE> row_of(const AttnArgs& a, const Item& it, const Range& rg, int r)
{
    Row<TREE> x;
    x.there = r < rg.rows;
    const int tok = x.there ? token_of(a, r) : 0;
    x.row = it.q.row0 + tok;
    x.head = it.head * a.G + (x.there ? r - tok * a.G : 0);
    const int p = rg.p0 + tok;
    x.sight.hi = !x.there ? 0 : (a.causal && p + 1 < rg.held ? p + 1 : rg.held);
    x.sight.lo = a.window > 0 ? p - a.window + 1 : 0;
    if constexpr (TREE) {
        if (x.sight.lo < 0) x.sight.lo = 0;      // (so that no difference of places leaves 32 bits)
        x.sight.row = -1;
        x.sight.p0 = rg.p0;
        x.sight.held = rg.held;
        if (is_tree<TREE>(a, it.q.n) && x.there) {
            x.sight.row = x.row;
            x.sight.hi = rg.p0 < rg.held ? rg.p0 : rg.held;
            if (a.window > 0) {      // (a position is one of the sequence's rows', whatever the tensor holds)
                const int at = a.positions[x.row], last = it.q.kv - 1;
                const int lo = (at < rg.p0 ? rg.p0 : at > last ? last : at) - a.window + 1;
                x.sight.lo = lo < 0 ? 0 : lo;
            }
        }
    }
    return x;
}

// Entries of a sequence's page table, 64 at a time, one to a lane; an entry that names no page, or lies past `end`, is -1.
struct Entries {
    int base = 0, id = -1;
    __device__ __forceinline__ void hold(const KVView& c, int seq, int page, int end)
    {
        base = page;
        const int p = page + lane_id();
        int v = -1;
        if (p < c.max_pages && ((int64_t)p << c.page_shift) < end) v = c.table[(int64_t)seq * c.max_pages + p];
        id = v >= 0 && v < c.n_pages ? v : -1;
    }
};

// N consecutive dwords, as wide as they can be loaded.  STREAM: bytes that nobody asks for again.
typedef uint32_t uint32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t uint32x4_t __attribute__((ext_vector_type(4)));
template <bool STREAM, typename V> __device__ __forceinline__ V load_as(const char* p)
{
    if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
    else return *reinterpret_cast<const V*>(p);
}
template <bool STREAM = false, int N> __device__ __forceinline__ void load_dwords(const char* p, uint32_t (&x)[N])
{
    if constexpr (N == 1) {
        x[0] = load_as<STREAM, uint32_t>(p);
    } else if constexpr (N == 2) {
        const uint32x2_t v = load_as<STREAM, uint32x2_t>(p);
        x[0] = v.x; x[1] = v.y;
    } else {
        static_assert(N % 4 == 0, "whole 16-byte pieces");
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const uint32x4_t v = load_as<STREAM, uint32x4_t>(p + 16 * i);
            x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
        }
    }
}

// What turns a row's sums into its result: the factor of its outputs, and its log-sum-exp.
struct Finish {
    float factor, lse;
};
__device__ __forceinline__ Finish finish_row(const AttnArgs& a, int head, float m, float l)
{
    Finish f;
    f.factor = 1.0f;
    if (a.sinks) {
        const float s2 = a.sinks[head] * kLog2e;
        const float m2 = fmaxf(m, s2);
        f.factor = __builtin_amdgcn_exp2f(m - m2);
        l = l * f.factor + __builtin_amdgcn_exp2f(s2 - m2);
        m = m2;
    }
    f.factor = l == 0.0f ? 0.0f : f.factor / l;
    f.lse = l == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
    return f;
}
// Four dimensions from d on of a finished row.
template <typename T> __device__ __forceinline__ void store_out(const AttnArgs& a, int row, int head, int D, int d, float4 o)
{
    T* dst = static_cast<T*>(a.out) + (int64_t)row * a.ldo + head * D + d;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(o.x, o.y), pack_bf16x2(o.z, o.w));
    else *reinterpret_cast<float4*>(dst) = o;
}

// ---- partial results of a piece: per row its output sums, maximum and sum, to be read by the block that ends the tile ----
// Like store_shared and load_shared, 16 bytes at a time: past the caches of one XCD (the buffer instructions take that as a constant,
// and keep to the workspace by themselves).
constexpr int kShared = 1 << 4;      // sc1
struct Parts {
    __amdgpu_buffer_rsrc_t sums;
    int D;
};
__device__ __forceinline__ Parts parts_of(const AttnArgs& a, int D)
{
    return Parts{__builtin_amdgcn_make_buffer_rsrc(a.part, 0, kPartUnits * 16 * D * (int)sizeof(float), 0x00020000), D};
}
__device__ __forceinline__ void store_part(const Parts& p, int row, int d, float4 o)
{
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uint32x4_t, o), p.sums, (row * p.D + d) * (int)sizeof(float), 0, kShared);
}
__device__ __forceinline__ float4 load_part(const Parts& p, int row, int d)
{
    return __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(p.sums, (row * p.D + d) * (int)sizeof(float), 0, kShared));
}
__device__ __forceinline__ void store_part_stats(const AttnArgs& a, int row, float m, float l)
{
    store_shared(reinterpret_cast<uint64_t*>(a.part_stats + row), (uint64_t)__float_as_uint(m) | (uint64_t)__float_as_uint(l) << 32);
}
__device__ __forceinline__ float2 load_part_stats(const AttnArgs& a, int row)
{
    const uint64_t v = load_shared(reinterpret_cast<const uint64_t*>(a.part_stats + row));
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// Every thread of a block that has stored its piece of a tile calls it; the block that ends the tile joins its pieces, in their order (so
// the result does not depend on who came last).  Sixteen lanes to a row, four pieces in flight.
template <typename T, int DP, int UNITS, bool TREE>
__device__ __forceinline__ void join_pieces(const AttnArgs& a, const Item& it, const Range& rg, int D, int32_t* flag)
{
    if (!last_to_arrive(a.tickets + it.slot, (uint32_t)rg.pieces, flag)) return;
    constexpr int ND = (DP + 63) / 64, AT_ONCE = UNITS == 1 || ND == 4 ? 1 : 4 / ND < UNITS ? 4 / ND : UNITS;      // units, as many as 64 registers hold
    const int units = it.q.units, d0 = (threadIdx.x & 15) * 4, q = threadIdx.x >> 4;
    const Parts parts = parts_of(a, D);
    for (int u0 = 0; u0 < units; u0 += AT_ONCE) {
        if (rg.first + u0 * 16 >= rg.rows) return;
        float M[AT_ONCE], L[AT_ONCE];
        float4 o[AT_ONCE][ND];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            M[u] = kLowest;
            L[u] = 0;
#pragma unroll
            for (int k = 0; k < ND; ++k) o[u][k] = make_float4(0, 0, 0, 0);
        }
        for (int c0 = 0; c0 < rg.pieces; c0 += 4) {
            float2 st[4][AT_ONCE];
            float4 x[4][AT_ONCE][ND];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (c0 + c < rg.pieces) {
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u) {
                        const int row = (it.slot + (c0 + c) * units + u0 + u) * 16 + q;
                        st[c][u] = load_part_stats(a, row);
#pragma unroll
                        for (int k = 0; k < ND; ++k) x[c][u][k] = load_part(parts, row, d0 + k * 64 < D ? d0 + k * 64 : 0);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                float top = M[u];
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (c0 + c < rg.pieces) top = fmaxf(top, st[c][u].x);
                const float back = __builtin_amdgcn_exp2f(M[u] - top);
                M[u] = top;
                L[u] *= back;
#pragma unroll
                for (int k = 0; k < ND; ++k) { o[u][k].x *= back; o[u][k].y *= back; o[u][k].z *= back; o[u][k].w *= back; }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if (c0 + c < rg.pieces) {
                        const float f = __builtin_amdgcn_exp2f(st[c][u].x - top);
                        L[u] += st[c][u].y * f;
#pragma unroll
                        for (int k = 0; k < ND; ++k) {
                            const float4 v = x[c][u][k];
                            o[u][k].x += v.x * f; o[u][k].y += v.y * f; o[u][k].z += v.z * f; o[u][k].w += v.w * f;
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const auto row = row_of<TREE>(a, it, rg, rg.first + (u0 + u) * 16 + q);
            if (!row.there || u0 + u >= units) continue;
            const Finish f = finish_row(a, row.head, M[u], L[u]);
#pragma unroll
            for (int k = 0; k < ND; ++k)
                if (d0 + k * 64 < D)
                    store_out<T>(a, row.row, row.head, D, d0 + k * 64, make_float4(o[u][k].x * f.factor, o[u][k].y * f.factor, o[u][k].z * f.factor, o[u][k].w * f.factor));
            if (a.lse && d0 == 0) a.lse[(int64_t)row.row * a.Hq + row.head] = f.lse;
        }
    }
}

}  // namespace
}  // namespace moe
