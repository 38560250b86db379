// Attention of a batch's new rows to a paged key/value cache.
//
// For a row q of a head, over the tokens j it sees:  x_j = (q . k_j) log2(e) / sqrt(dim),  out = sum_j 2^(x_j - M) v_j / sum_j 2^(x_j - M),
// in one pass over the tokens with a running M and sum (a later maximum scales what has been summed so far).  The rows of all
// query heads that read one key/value head are one matrix: packed row r of a sequence is new token r / G, query head h G + r % G.
//
// Work is cut on the device, from the descriptors: every block of a launch reads them and finds its own item (sequence, key/value
// head, tile of packed rows, piece of the history), so no host ever waits for a length.  Pieces are as long as spreads the batch's work over
// the chip; a row whose history is in several pieces is joined by a second launch from fp32 partial results.
#include "kv.h"

#include <cfloat>

namespace moe {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float float4_t __attribute__((ext_vector_type(4)));

constexpr float kLowest = -FLT_MAX;      // a running maximum before its first token: finite, so that no difference is NaN
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// ----------------------------------------------------------------------------------------------------------------
// The plan.
// ----------------------------------------------------------------------------------------------------------------
constexpr int kItems = 2048;        // items that the pieces of a launch aim at
constexpr int kMinPiece = 128;      // tokens: a step of 32 (fp32: of 16 or more) for each of a block's four waves

struct Seq {
    int row0, n, kv;                // first row, rows, tokens held
    int tiles, units, len;          // tiles of packed rows, units of 16 rows to a tile, tokens of the longest tile's range
};
struct Item {
    Seq q;
    int seq, head, tile, sub;       // sub: the piece (or, in the joining launch, the unit of 16 rows)
    int piece;                      // tokens of a piece; 0: the history is in one
    int slot;                       // of the partial results: first unit of the tile's first piece
    bool valid;
};

__device__ __forceinline__ Seq shape_of(const AttnArgs& a, int lo, int hi, int kv)
{
    Seq q;
    lo = lo < 0 ? 0 : (lo > a.c.T ? a.c.T : lo);
    hi = hi < lo ? lo : (hi > a.c.T ? a.c.T : hi);
    const int64_t most = (int64_t)a.c.max_pages << a.c.page_shift;
    kv = kv < 0 ? 0 : ((int64_t)kv > most ? (int)most : kv);
    q.row0 = lo;
    q.n = hi - lo;
    q.kv = kv;
    const int rows = q.n * a.G;
    q.units = rows <= 16 ? 1 : a.tile_rows / 16;
    q.tiles = rows <= 16 ? (rows > 0 ? 1 : 0) : (rows + a.tile_rows - 1) / a.tile_rows;
    q.len = kv;
    if (a.window > 0) {
        int first = kv - q.n - a.window + 1;
        q.len = kv - (first > 0 ? first : 0) + 31;
        const int64_t w = (int64_t)a.window + a.tile_rows / a.G + 2 + 31;
        if (a.causal && w < q.len) q.len = (int)w;
        if (q.len > kv) q.len = kv;
    }
    return q;
}

// The item of block `block`.  JOIN: the block's unit of 16 rows among those whose history is in several pieces.
// Sequences are taken 256 at a time, four to a lane.  A sequence whose partial results no longer fit the workspace stays in one piece.
template <bool JOIN> __device__ __forceinline__ Item find_item(const AttnArgs& a, int block)
{
    const int lane = lane_id();
    const int S = a.c.S, Hk = a.c.Hk;
    Seq q[4];
    auto load = [&](int b) {
        int off[5], kv[4];
#pragma unroll
        for (int i = 0; i < 5; ++i) {
            const int s = b + lane * 4 + i;
            off[i] = a.c.off[s < S ? s : S];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = b + lane * 4 + i;
            kv[i] = a.c.lens[s < S ? s : S - 1];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = shape_of(a, off[i], b + lane * 4 + i < S ? off[i + 1] : off[i], kv[i]);
    };
    float work = 0;
    for (int b = 0; b < S; b += 256) {
        load(b);
#pragma unroll
        for (int i = 0; i < 4; ++i) work += (float)q[i].tiles * (float)q[i].len;
    }
    work = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wave_scan(work)), 63)) * (float)Hk;
    int piece = kMinPiece;
    const float even = work * (1.0f / kItems);
    if (even > (float)piece) piece = even < 1e9f ? ((int)even + kMinPiece) / kMinPiece * kMinPiece : 1 << 30;

    Item it;
    it.valid = false;
    int items0 = 0;
    float slots0 = 0;               // (as floats: they only grow, and past the workspace only that counts)
    for (int b = 0; b < S; b += 256) {
        if (S > 256) load(b);
        int pieces[4];
        float want = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            pieces[i] = (int)(((int64_t)q[i].len + piece - 1) / piece);
            if (pieces[i] < 1) pieces[i] = 1;
            want += pieces[i] > 1 ? (float)q[i].tiles * Hk * pieces[i] * q[i].units : 0.0f;
        }
        const float incl = wave_scan(want);
        float at = slots0 + incl - want;
        int mine = 0, slot[4], count[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float need = pieces[i] > 1 ? (float)q[i].tiles * Hk * pieces[i] * q[i].units : 0.0f;
            slot[i] = 0;
            if (need > 0) {
                if (at + need <= (float)kPartUnits) slot[i] = (int)at;
                else pieces[i] = 1;
            }
            at += need;
            count[i] = JOIN ? (pieces[i] > 1 ? q[i].tiles * Hk * q[i].units : 0) : q[i].tiles * Hk * pieces[i];
            mine += count[i];
        }
        slots0 += __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, incl), 63));
        const int incl_items = items0 + wave_scan(mine);
        const unsigned long long hit = __ballot(block < incl_items);
        if (hit != 0) {
            const int src = __ffsll((long long)hit) - 1;
            int rem = block - (incl_items - mine);
            int seq = 0, sl = 0, pc = 1;
            Seq f = q[0];
            bool found = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!found && rem < count[i]) {
                    found = true;
                    f = q[i];
                    seq = b + lane * 4 + i;
                    sl = slot[i];
                    pc = pieces[i];
                } else if (!found) {
                    rem -= count[i];
                }
            }
            auto pick = [&](int v) { return __builtin_amdgcn_readlane(v, src); };
            it.q.row0 = pick(f.row0); it.q.n = pick(f.n); it.q.kv = pick(f.kv);
            it.q.tiles = pick(f.tiles); it.q.units = pick(f.units); it.q.len = pick(f.len);
            it.seq = pick(seq);
            rem = pick(rem);
            sl = pick(sl);
            pc = pick(pc);
            // heads side by side (they go to different XCDs, and the tiles of a head to the same ones), long tiles first
            const int per = JOIN ? it.q.units : pc;
            it.head = rem % Hk;
            rem /= Hk;
            it.sub = rem % per;
            it.tile = it.q.tiles - 1 - rem / per;
            it.piece = pc > 1 ? piece : 0;
            it.slot = sl + (it.tile * Hk + it.head) * pc * it.q.units;
            it.valid = rem >= 0 && it.tile >= 0;      // (always, but for descriptors so wrong that the counts overflow)
            return it;
        }
        items0 = __builtin_amdgcn_readlane(incl_items, 63);
    }
    return it;
}

// The tokens that a tile's rows see: all rows those of [full_lo, full_hi), some row those of [lo, hi); lo is a multiple of 32.
struct Range {
    int p0;                         // position of the sequence's first row
    int lo, hi, full_lo, full_hi;
    int pieces;
};
__device__ __forceinline__ Range range_of(const AttnArgs& a, const Item& it)
{
    const int rows = it.q.n * a.G;
    const int first = it.tile * it.q.units * 16;
    const int end = first + it.q.units * 16;
    const int last = (end < rows ? end : rows) - 1;
    Range r;
    r.p0 = it.q.kv - it.q.n;
    const int p_first = r.p0 + first / a.G, p_last = r.p0 + last / a.G;
    r.hi = a.causal && p_last + 1 < it.q.kv ? p_last + 1 : it.q.kv;
    if (r.hi < 0) r.hi = 0;
    r.full_hi = a.causal && p_first + 1 < it.q.kv ? p_first + 1 : it.q.kv;
    r.lo = a.window > 0 && p_first - a.window + 1 > 0 ? p_first - a.window + 1 : 0;
    r.full_lo = a.window > 0 && p_last - a.window + 1 > 0 ? p_last - a.window + 1 : 0;
    r.lo &= ~31;
    const int len = r.hi > r.lo ? r.hi - r.lo : 0;
    r.pieces = it.piece > 0 && len > it.piece ? (len + it.piece - 1) / it.piece : 1;
    return r;
}

// Maximum and sum over the four lanes that hold the tokens of one row (lanes l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float max_over_tokens(float v)
{
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float sum_over_tokens(float v)
{
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// N consecutive dwords, as wide as they can be loaded.
template <int N> __device__ __forceinline__ void load_dwords(const char* p, uint32_t (&x)[N])
{
    if constexpr (N == 1) {
        x[0] = *reinterpret_cast<const uint32_t*>(p);
    } else if constexpr (N == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        x[0] = v.x; x[1] = v.y;
    } else {
        static_assert(N % 4 == 0, "whole 16-byte pieces");
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const uint4 v = reinterpret_cast<const uint4*>(p)[i];
            x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
        }
    }
}

// out = o / l of a finished row, 4 dimensions of it, with the head's sink.
template <typename T>
__device__ __forceinline__ void store_row(const AttnArgs& a, int row, int head, int d, const float (&o)[4], float m, float l)
{
    if (a.sinks) {
        const float s2 = a.sinks[head] * kLog2e;
        const float m2 = fmaxf(m, s2);
        const float f = __builtin_amdgcn_exp2f(m - m2);
        l = l * f + __builtin_amdgcn_exp2f(s2 - m2);
        m = m2;
        const float g = l == 0.0f ? 0.0f : f / l;
        T* dst = static_cast<T*>(a.out) + (int64_t)row * a.ldo + head * a.c.D + d;
        if constexpr (sizeof(T) == 2)
            *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(o[0] * g, o[1] * g), pack_bf16x2(o[2] * g, o[3] * g));
        else
            *reinterpret_cast<float4*>(dst) = make_float4(o[0] * g, o[1] * g, o[2] * g, o[3] * g);
    } else {
        const float g = l == 0.0f ? 0.0f : 1.0f / l;
        T* dst = static_cast<T*>(a.out) + (int64_t)row * a.ldo + head * a.c.D + d;
        if constexpr (sizeof(T) == 2)
            *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(o[0] * g, o[1] * g), pack_bf16x2(o[2] * g, o[3] * g));
        else
            *reinterpret_cast<float4*>(dst) = make_float4(o[0] * g, o[1] * g, o[2] * g, o[3] * g);
    }
    if (a.lse && d == 0)
        a.lse[(int64_t)row * a.Hq + head] = l == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ----------------------------------------------------------------------------------------------------------------
// The kernel for few rows: keys and values go from memory to the matrix cores' registers, through no LDS.
//
// A wave takes TOK tokens at a time for up to NQ * 16 rows.  Scores are computed transposed, S = K Q^T, and so is the output,
// O = V^T P^T: a lane then holds, in both products, column q = lane % 16, so a row's maximum, sum and scale are lane-local
// but for two exchanges a step, and the exponentials it has computed are, as they stand, its operand of the second product
// (a contraction may take its tokens in any order; here lane group g = lane / 16 has tokens 4 g .. 4 g + 3 of each 16).
// K is read as the operand wants it, 16 bytes of a token's row to a lane; V in whole rows, DP / 16 dimensions to a lane, and
// eight tokens' dwords are put together by byte permutes, which is all the transposing there is.
// The four waves of a block take a quarter of the piece each and join through LDS.
// ----------------------------------------------------------------------------------------------------------------
template <typename T, bool FP8, int DP, int NQ> struct Few {
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int NJ = F32 ? 1 : 2, TOK = NJ * 16;          // 16-token subtiles of a step
    static constexpr int ESZ = FP8 ? 1 : (int)sizeof(T);
    static constexpr int KC = DP / (F32 ? 16 : (FP8 ? 64 : 32));   // key loads per subtile
    static constexpr int KDIM = F32 ? 4 : (FP8 ? 16 : 8);          // dimensions of such a load
    static constexpr int KDW = KDIM * ESZ / 4;
    static constexpr int VW = DP / 16, VDW = VW * ESZ / 4;         // dimensions and dwords of a token's values in a lane
    static constexpr int LDR = DP + 4;                             // floats of a row in LDS

    struct Shared {
        float stats[2][4][NQ * 16];
        float o[4][16][LDR];
    };

    // The queries as the first product's second operand; zeros past the dimension and for rows that are not there.
    struct Queries {
        bf16x8_t b[F32 ? 1 : NQ][F32 ? 1 : DP / 32];
        float f[F32 ? NQ : 1][F32 ? DP / 16 : 1][4];
    };

    static __device__ __forceinline__ void run(const AttnArgs& a, const Item& it, Shared& sh)
    {
        const Range rg = range_of(a, it);
        if (it.sub >= rg.pieces) return;
        const int lane = lane_id(), n = lane & 15, g = lane >> 4;
        const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
        const int D = a.c.D, shift = a.c.page_shift, Hk = a.c.Hk;
        const int rows = it.q.n * a.G, first = it.tile * NQ * 16;

        int begin = rg.lo, end = rg.hi;
        if (rg.pieces > 1) {
            begin += it.sub * it.piece;
            if (end - begin > it.piece) end = begin + it.piece;
        }
        const int per = end > begin ? (end - begin + 4 * TOK - 1) / (4 * TOK) * TOK : 0;
        const int t0 = begin + wave * per;
        const int t1 = t0 + per < end ? t0 + per : end;

        // rows: what each sees, and its queries
        int see_lo[NQ], see_hi[NQ];
        Queries Q;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const int r = first + i * 16 + n;
            const bool there = r < rows;
            const int tok = there ? r / a.G : 0, hd = it.head * a.G + (there ? r - tok * a.G : 0);
            const int p = rg.p0 + tok;
            see_hi[i] = !there ? 0 : (a.causal && p + 1 < it.q.kv ? p + 1 : it.q.kv);
            see_lo[i] = a.window > 0 ? p - a.window + 1 : 0;
            const T* src = static_cast<const T*>(a.q) + (int64_t)(it.q.row0 + tok) * a.ldq + (int64_t)hd * D;
            if constexpr (F32) {
#pragma unroll
                for (int c = 0; c < DP / 16; ++c) {
                    const int d = c * 16 + g * 4;
                    const float4 v = *reinterpret_cast<const float4*>(src + (d < D ? d : 0));
                    const float z = there && d < D ? 1.0f : 0.0f;
                    Q.f[i][c][0] = z != 0 ? v.x : 0; Q.f[i][c][1] = z != 0 ? v.y : 0;
                    Q.f[i][c][2] = z != 0 ? v.z : 0; Q.f[i][c][3] = z != 0 ? v.w : 0;
                }
            } else {
#pragma unroll
                for (int c = 0; c < DP / 32; ++c) {
                    const int d = FP8 ? (c / 2) * 64 + g * 16 + (c % 2) * 8 : c * 32 + g * 8;
                    uint4 v = *reinterpret_cast<const uint4*>(src + (d < D ? d : 0));
                    if (!there || d >= D) v = make_uint4(0, 0, 0, 0);
                    Q.b[i][c] = __builtin_bit_cast(bf16x8_t, v);
                }
            }
        }

        float m[NQ], l[NQ];
        float4_t o[VDW][NQ][PER];      // dimension (row of the output tile) * VW + x * PER + y
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            m[i] = kLowest;
            l[i] = 0;
#pragma unroll
            for (int f = 0; f < VW; ++f) o[f / PER][i][f % PER] = float4_t{0, 0, 0, 0};
        }

        // 64 entries of the page table at a time, one to a lane; an entry that names no page is -1
        int base = 0, entries = -1;
        auto hold = [&](int page) {
            base = page;
            const int p = page + lane;
            int id = -1;
            if (p < a.c.max_pages && ((int64_t)p << shift) < t1) id = a.c.table[(int64_t)it.seq * a.c.max_pages + p];
            entries = id >= 0 && id < a.c.n_pages ? id : -1;
        };
        auto page_of = [&](int t) { return __shfl(entries, (t >> shift) - base); };
        auto row_of = [&](int id, int t) {
            return page_row(id < 0 ? 0 : id, Hk, it.head, shift, t & ((1 << shift) - 1));
        };

        // a step's loads: keys of token 16 j + n, values of tokens 16 j + 4 g + r
        uint32_t kr[NJ][KC][KDW], vr[VDW][NJ * 4];
        uint32_t ks[NJ], vs[NJ];
        int vid[NJ];                 // page of this lane's four tokens of a subtile
        auto load_k = [&](int t) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int tok = t + j * 16 + n;
                const int64_t row = row_of(page_of(tok), tok);
                const char* p = a.c.k + row * D * ESZ;
#pragma unroll
                for (int c = 0; c < KC; ++c) {
                    const int d = c * (4 * KDIM) + g * KDIM;
                    load_dwords(p + (d < D ? d : 0) * ESZ, kr[j][c]);      // (past the dimension the queries are zero)
                }
                if constexpr (FP8) ks[j] = a.c.ks[row];
            }
        };
        auto load_v = [&](int t) {
            const int d = n * VW < D ? n * VW : 0;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int tok = t + j * 16 + g * 4;
                vid[j] = page_of(tok);
                const int64_t row = row_of(vid[j], tok);
                const char* p = a.c.v + (row * D + d) * ESZ;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    uint32_t raw[VDW];
                    load_dwords(p + (int64_t)r * D * ESZ, raw);
#pragma unroll
                    for (int x = 0; x < VDW; ++x) vr[x][j * 4 + r] = raw[x];
                }
                if constexpr (FP8) vs[j] = *reinterpret_cast<const uint32_t*>(a.c.vs + row);
            }
        };

        if (t0 < t1) {
            hold(t0 >> shift);
            load_k(t0);
            load_v(t0);
        }
        for (int t = t0; t < t1; t += TOK) {
            const bool more = t + TOK < t1;
            float4_t s[NQ][NJ];
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
#pragma unroll
                for (int i = 0; i < NQ; ++i) s[i][j] = float4_t{0, 0, 0, 0};
                if constexpr (F32) {
#pragma unroll
                    for (int c = 0; c < KC; ++c) {
                        float kf[4];
                        if constexpr (FP8) {
                            const hw_float2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)kr[j][c][0], false);
                            const hw_float2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)kr[j][c][0], true);
                            kf[0] = lo[0]; kf[1] = lo[1]; kf[2] = hi[0]; kf[3] = hi[1];
                        } else {
#pragma unroll
                            for (int x = 0; x < 4; ++x) kf[x] = __uint_as_float(kr[j][c][x]);
                        }
#pragma unroll
                        for (int x = 0; x < 4; ++x)
#pragma unroll
                            for (int i = 0; i < NQ; ++i)
                                s[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[x], Q.f[i][c][x], s[i][j], 0, 0, 0);
                    }
                } else {
                    float sc = 1.0f;
                    if constexpr (FP8) sc = scale_of(ks[j]);
#pragma unroll
                    for (int c = 0; c < KC; ++c)
#pragma unroll
                        for (int x = 0; x < KDW / (FP8 ? 2 : 4); ++x) {
                            bf16x8_t kb;
                            if constexpr (FP8) {        // exact: a code has 4 significant bits, its scale is a power of two
#pragma unroll
                                for (int w = 0; w < 2; ++w) {
                                    const uint32_t codes = kr[j][c][x * 2 + w];
                                    const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, sc, false);
                                    const bf16x2_t hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, sc, true);
                                    kb[w * 4] = lo[0]; kb[w * 4 + 1] = lo[1]; kb[w * 4 + 2] = hi[0]; kb[w * 4 + 3] = hi[1];
                                }
                            } else {
                                kb = __builtin_bit_cast(bf16x8_t, kr[j][c]);
                            }
#pragma unroll
                            for (int i = 0; i < NQ; ++i)
                                s[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, Q.b[i][c * (FP8 ? 2 : 1) + x], s[i][j], 0, 0, 0);
                        }
                }
            }
            // (the fp32 path applies a key's scale to its score, a lane of which holds tokens 4 g + r)
            float kscale[NJ][4];
            if constexpr (F32 && FP8) {
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) kscale[j][r] = scale_of((uint32_t)__shfl((int)ks[j], g * 4 + r));
            }
            if (more) {
                if (((t + 2 * TOK - 1) >> shift) - base >= 64) hold((t + TOK) >> shift);
                load_k(t + TOK);
            }

            bool gone = false;
#pragma unroll
            for (int j = 0; j < NJ; ++j) gone |= vid[j] < 0;
            const bool masked = t + TOK > rg.full_hi || t + TOK > end || t < rg.full_lo || __any(gone);
            float p[NQ][NJ][4];
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                float top = -__builtin_inff();
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float x = s[i][j][r] * a.scale2;
                        if constexpr (F32 && FP8) x *= kscale[j][r];
                        if (masked) {
                            const int tok = t + j * 16 + g * 4 + r;
                            if (!(vid[j] >= 0 && tok < see_hi[i] && tok >= see_lo[i])) x = -__builtin_inff();
                        }
                        p[i][j][r] = x;
                        top = fmaxf(top, x);
                    }
                top = max_over_tokens(top);
                // The reference of the exponentials follows the maximum only when that has grown by more than 8: until then they stay below
                // 2^8, which fp32 sums and bf16 weights hold as well as values below 1.
                if (__any(top > m[i] + 8.0f)) {
                    const float to = fmaxf(top, m[i]), f = __builtin_amdgcn_exp2f(m[i] - to);
                    m[i] = to;
                    l[i] *= f;
#pragma unroll
                    for (int x = 0; x < VW; ++x) o[x / PER][i][x % PER] *= f;
                }
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        p[i][j][r] = __builtin_amdgcn_exp2f(p[i][j][r] - m[i]);
                        l[i] += p[i][j][r];
                    }
            }
            // values: tokens that no row sees are zeros, whatever the page holds
            if (masked) {
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const bool none = vid[j] < 0 || t + j * 16 + g * 4 + r >= rg.hi;
                        if (none) {
#pragma unroll
                            for (int x = 0; x < VDW; ++x) vr[x][j * 4 + r] = 0;
                        }
                        if constexpr (FP8) {
                            if (none) vs[j] = (vs[j] & ~(255u << (8 * r))) | (127u << (8 * r));
                        }
                    }
                strange_values(t, see_lo, see_hi, vid, vr, vs, o);
            }
            if constexpr (FP8) {        // a value's scale goes to its weight: exact, and one product instead of dim
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float sc = scale_of((vs[j] >> (8 * r)) & 255u);
#pragma unroll
                        for (int i = 0; i < NQ; ++i) p[i][j][r] *= sc;
                    }
            }
            const Weights w = weights_of(p);
#pragma unroll
            for (int x = 0; x < VDW; ++x) add_values(vr[x], w, o[x]);
            if (more) load_v(t + TOK);
        }

        // a wave's sums, then the block's
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            l[i] = sum_over_tokens(l[i]);
            if (g == 0) {
                sh.stats[0][wave][i * 16 + n] = m[i];
                sh.stats[1][wave][i * 16 + n] = l[i];
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            float top = kLowest;
#pragma unroll
            for (int w = 0; w < 4; ++w) top = fmaxf(top, sh.stats[0][w][i * 16 + n]);
            const float f = __builtin_amdgcn_exp2f(m[i] - top);
            if (i > 0) __syncthreads();
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float* dst = &sh.o[wave][n][(g * 4 + r) * VW];
                auto out = [&](int x) { return o[x / PER][i][x % PER][r] * f; };
#pragma unroll
                for (int x = 0; x < VW / 4; ++x)
                    reinterpret_cast<float4*>(dst)[x] = make_float4(out(4 * x), out(4 * x + 1), out(4 * x + 2), out(4 * x + 3));
            }
            __syncthreads();
            const int q = threadIdx.x >> 4, r = first + i * 16 + q;
            if (r < rows) {
                float M = kLowest, L = 0;
#pragma unroll
                for (int w = 0; w < 4; ++w) M = fmaxf(M, sh.stats[0][w][i * 16 + q]);
#pragma unroll
                for (int w = 0; w < 4; ++w) L += sh.stats[1][w][i * 16 + q] * __builtin_amdgcn_exp2f(sh.stats[0][w][i * 16 + q] - M);
                const int tok = r / a.G, hd = it.head * a.G + (r - tok * a.G);
                const int64_t unit = it.slot + it.sub * it.q.units + i;
                if (rg.pieces > 1 && (threadIdx.x & 15) == 0) a.part_stats[unit * 16 + q] = make_float2(M, L);
                for (int d = (threadIdx.x & 15) * 4; d < D; d += 64) {
                    float v[4] = {};
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float4 x = *reinterpret_cast<const float4*>(&sh.o[w][q][d]);
                        v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
                    }
                    if (rg.pieces > 1)
                        *reinterpret_cast<float4*>(a.part + (unit * 16 + q) * D + d) = make_float4(v[0], v[1], v[2], v[3]);
                    else
                        store_row<T>(a, it.q.row0 + tok, hd, d, v, M, L);
                }
            }
        }
    }

    // The weights as the second product's operand.
    struct Weights {
        bf16x8_t b[F32 ? 1 : NQ];
        float f[F32 ? NQ : 1][4];
    };
    static __device__ __forceinline__ Weights weights_of(const float (&p)[NQ][NJ][4])
    {
        Weights w;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if constexpr (F32) {
#pragma unroll
                for (int r = 0; r < 4; ++r) w.f[i][r] = p[i][0][r];
            } else {
                const uint4 u = make_uint4(pack_bf16x2(p[i][0][0], p[i][0][1]), pack_bf16x2(p[i][0][2], p[i][0][3]),
                                           pack_bf16x2(p[i][NJ - 1][0], p[i][NJ - 1][1]), pack_bf16x2(p[i][NJ - 1][2], p[i][NJ - 1][3]));
                w.b[i] = __builtin_bit_cast(bf16x8_t, u);
            }
        }
        return w;
    }

    // Output tiles += values x weights, for one dword of every token's values: PER dimensions.
    static constexpr int PER = VW / VDW;
    static __device__ __forceinline__ void add_values(const uint32_t (&v)[NJ * 4], const Weights& w, float4_t (&o)[NQ][PER])
    {
        if constexpr (F32) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float vf[4] = {__uint_as_float(v[r]), 0, 0, 0};
                if constexpr (FP8) {
                    const hw_float2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[r], false);
                    const hw_float2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)v[r], true);
                    vf[0] = lo[0]; vf[1] = lo[1]; vf[2] = hi[0]; vf[3] = hi[1];
                }
#pragma unroll
                for (int y = 0; y < PER; ++y)
#pragma unroll
                    for (int i = 0; i < NQ; ++i) o[i][y] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[y], w.f[i][r], o[i][y], 0, 0, 0);
            }
        } else {
            uint32_t f[PER][4];          // [dimension][token pair], bf16 pairs
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (FP8) {
                    const uint32_t lo = __builtin_amdgcn_perm(v[2 * k + 1], v[2 * k], 0x05010400u);
                    const uint32_t hi = __builtin_amdgcn_perm(v[2 * k + 1], v[2 * k], 0x07030602u);
                    f[0][k] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
                    f[1][k] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
                    f[2][k] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
                    f[3][k] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
                } else {
                    f[0][k] = __builtin_amdgcn_perm(v[2 * k + 1], v[2 * k], 0x05040100u);
                    f[1][k] = __builtin_amdgcn_perm(v[2 * k + 1], v[2 * k], 0x07060302u);
                }
            }
#pragma unroll
            for (int y = 0; y < PER; ++y) {
                const bf16x8_t vb = __builtin_bit_cast(bf16x8_t, f[y]);
#pragma unroll
                for (int i = 0; i < NQ; ++i) o[i][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, w.b[i], o[i][y], 0, 0, 0);
            }
        }
    }

    // Values that are not finite, in a step whose tokens not every row sees: a weight of zero would not keep them out of the
    // sums.  They are taken out of vr; rows that see one get it as the infinity or NaN that it is.
    static __device__ __forceinline__ void strange_values(int t, const int (&see_lo)[NQ], const int (&see_hi)[NQ], const int (&vid)[NJ],
                                                          uint32_t (&vr)[VDW][NJ * 4], uint32_t (&vs)[NJ], float4_t (&o)[VDW][NQ][PER])
    {
        const int g = lane_id() >> 4;
        // kind of value y of a dword of slot s: 0 finite, 1 inf, 2 -inf, 3 NaN
        auto kind = [&](uint32_t dword, int s, int y) -> int {
            if constexpr (FP8) {
                const bool nan_scale = ((vs[s / 4] >> (8 * (s % 4))) & 255u) == 255u;
                return nan_scale || ((dword >> (8 * y)) & 0x7fu) == 0x7fu ? 3 : 0;
            } else if constexpr (F32) {
                return (dword & 0x7f800000u) != 0x7f800000u ? 0 : (dword & 0x7fffffu) ? 3 : (dword >> 31) ? 2 : 1;
            } else {
                const uint32_t u = (dword >> (16 * y)) & 0xffffu;
                return (u & 0x7f80u) != 0x7f80u ? 0 : (u & 0x7fu) ? 3 : (u >> 15) ? 2 : 1;
            }
        };
        bool any = false;
#pragma unroll
        for (int x = 0; x < VDW; ++x)
#pragma unroll
            for (int s = 0; s < NJ * 4; ++s)
#pragma unroll
                for (int y = 0; y < PER; ++y) any |= kind(vr[x][s], s, y) != 0;
        if (!__any(any)) return;
        // 1 where a row sees a token, as weights
        float seen[NQ][NJ][4];
#pragma unroll
        for (int i = 0; i < NQ; ++i)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int tok = t + j * 16 + g * 4 + r;
                    seen[i][j][r] = vid[j] >= 0 && tok < see_hi[i] && tok >= see_lo[i] ? 1.0f : 0.0f;
                }
        const Weights w = weights_of(seen);
#pragma unroll
        for (int x = 0; x < VDW; ++x) {
#pragma unroll 1
            for (int what = 1; what <= 3; ++what) {
                uint32_t mark[NJ * 4];
#pragma unroll
                for (int s = 0; s < NJ * 4; ++s) {
                    mark[s] = 0;
#pragma unroll
                    for (int y = 0; y < PER; ++y)
                        if (kind(vr[x][s], s, y) == what) mark[s] |= (FP8 ? 0x38u : F32 ? 0x3f800000u : 0x3f80u) << (y * (32 / PER));
                }
                float4_t hits[NQ][PER];
#pragma unroll
                for (int i = 0; i < NQ; ++i)
#pragma unroll
                    for (int y = 0; y < PER; ++y) hits[i][y] = float4_t{0, 0, 0, 0};
                add_values(mark, w, hits);
                const float worth = what == 1 ? __builtin_inff() : what == 2 ? -__builtin_inff() : __builtin_nanf("");
#pragma unroll
                for (int i = 0; i < NQ; ++i)
#pragma unroll
                    for (int y = 0; y < PER; ++y)
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[x][i][y][r] += hits[i][y][r] > 0.5f ? worth : 0.0f;
            }
#pragma unroll
            for (int s = 0; s < NJ * 4; ++s) {
                uint32_t keep = 0;
#pragma unroll
                for (int y = 0; y < PER; ++y)
                    if (kind(vr[x][s], s, y) == 0) keep |= (0xffffffffu >> (32 - 32 / PER)) << (y * (32 / PER));
                vr[x][s] &= keep;
            }
        }
        if constexpr (FP8) {
#pragma unroll
            for (int s = 0; s < NJ * 4; ++s)
                if (((vs[s / 4] >> (8 * (s % 4))) & 255u) == 255u) vs[s / 4] = (vs[s / 4] & ~(255u << (8 * (s % 4)))) | (127u << (8 * (s % 4)));
        }
    }
};

template <typename T, bool FP8, int DP> __global__ __launch_bounds__(256, sizeof(T) == 4 || DP > 128 ? 1 : 2) void attention_kernel(AttnArgs a)
{
    constexpr int NQ = DP <= 128 ? 2 : 1;       // 32 rows of 256 dimensions do not fit the registers
    __shared__ union {
        typename Few<T, FP8, DP, 1>::Shared one;
        typename Few<T, FP8, DP, NQ>::Shared more;
    } sh;
    const Item it = find_item<false>(a, blockIdx.x);
    if (!it.valid) return;
    if (it.q.units == 1) Few<T, FP8, DP, 1>::run(a, it, sh.one);
    else if constexpr (NQ > 1) Few<T, FP8, DP, NQ>::run(a, it, sh.more);
}

// Joins the partial results of 16 packed rows: 16 lanes to a row.
template <typename T> __global__ __launch_bounds__(256) void join_kernel(AttnArgs a)
{
    const Item it = find_item<true>(a, blockIdx.x);
    if (!it.valid) return;
    const Range rg = range_of(a, it);
    if (rg.pieces < 2) return;
    const int rows = it.q.n * a.G;
    const int q = threadIdx.x >> 4, r = (it.tile * it.q.units + it.sub) * 16 + q;
    if (r >= rows) return;
    const int tok = r / a.G, hd = it.head * a.G + (r - tok * a.G), D = a.c.D;
    float M = kLowest, L = 0;
    for (int c = 0; c < rg.pieces; ++c) M = fmaxf(M, a.part_stats[(int64_t)(it.slot + c * it.q.units + it.sub) * 16 + q].x);
    for (int c = 0; c < rg.pieces; ++c) {
        const float2 st = a.part_stats[(int64_t)(it.slot + c * it.q.units + it.sub) * 16 + q];
        L += st.y * __builtin_amdgcn_exp2f(st.x - M);
    }
    for (int d = (threadIdx.x & 15) * 4; d < D; d += 64) {
        float v[4] = {};
        for (int c = 0; c < rg.pieces; ++c) {
            const int64_t at = (int64_t)(it.slot + c * it.q.units + it.sub) * 16 + q;
            const float f = __builtin_amdgcn_exp2f(a.part_stats[at].x - M);
            const float4 x = *reinterpret_cast<const float4*>(a.part + at * D + d);
            v[0] += x.x * f; v[1] += x.y * f; v[2] += x.z * f; v[3] += x.w * f;
        }
        store_row<T>(a, it.q.row0 + tok, hd, d, v, M, L);
    }
}

}  // namespace

hipError_t launch_attention(int dtype, bool fp8, AttnArgs a, hipStream_t s)
{
    a.tile_rows = a.c.D <= 128 ? 32 : 16;
    // tiles: a sequence has one, or as many as its packed rows fill; pieces: an item more each, kItems more in all
    const int64_t rows = (int64_t)a.c.T * a.G;
    const int64_t tiles = (a.c.S < a.c.T ? a.c.S : a.c.T) + rows / a.tile_rows;
    const int64_t base = tiles * a.c.Hk;
    const int64_t longest = (int64_t)a.c.max_pages << a.c.page_shift;
    const int64_t by_length = base * ((longest + kMinPiece - 1) / kMinPiece - 1);
    const int64_t more = by_length < kItems + 64 ? by_length : kItems + 64;
    if (base + more > 0x7fffffff) return hipErrorInvalidValue;
    const unsigned grid = (unsigned)(base + more);
    auto go = [&](auto t, auto f, auto dp) {
        attention_kernel<decltype(t), decltype(f)::value, decltype(dp)::value><<<grid, 256, 0, s>>>(a);
        return hipGetLastError();
    };
    auto by_dim = [&](auto t, auto f) {
        if (a.c.D <= 64) return go(t, f, std::integral_constant<int, 64>());
        if (a.c.D <= 128) return go(t, f, std::integral_constant<int, 128>());
        return go(t, f, std::integral_constant<int, 256>());
    };
    auto by_format = [&](auto t) { return fp8 ? by_dim(t, std::true_type()) : by_dim(t, std::false_type()); };
    hipError_t e = dtype == MOE_BF16 ? by_format(bf16_t()) : by_format(float());
    if (e != hipSuccess || more <= 0) return e;
    // every tile that is in pieces is among the first kItems of the work, and has two units at most
    const int64_t units = 2 * base < 2 * (kItems + 64) ? 2 * base : 2 * (kItems + 64);
    if (dtype == MOE_BF16) join_kernel<bf16_t><<<(unsigned)units, 256, 0, s>>>(a);
    else join_kernel<float><<<(unsigned)units, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace moe
