// The attention weight that cached tokens receive: column sums of exp(q . k / sqrt(dim) - lse), without the matrix they are sums of.
//
// Scores are computed transposed as in the attention, S = K Q^T, a query row to a lane's column: a row's lse is lane-local, and the sums of the
// exponentials over the rows stay in the lanes until the end.  There are three ways to bring rows and keys together, by the packed rows of a sequence:
//   up to 16: the rows stay in registers, and the keys stream by, read once, which bounds it.  64 rows over up to 8192 tokens, 188 MB of keys, 44 us,
//     4.3 TB/s (a copy of 4 GiB 4.8).  Keys are plain loads: an instruction takes half a line of each row (as a stream 54 -> 57 us).
//   up to what LDS holds (256; fp32 128): the rows stay there, and every wave takes 32 tokens' keys for itself, with no barrier until the end.
//     What bounds it: VALU, and the chain page table, keys, products of each 32 tokens.  32 rows of 64 heads over up to 16384 FP8 tokens in 12 sequences
//     44 us (61 as more rows are taken).  Sequences of fewer rows beside such, or beside prompts, are taken this way too.
//   more: a block holds 256 tokens' keys, 32 to a wave, and takes the rows that see them 128 at a time from LDS, brought there by direct
//     loads while the 128 before are used.  What bounds it: a prompt of 8192 rows and 32 heads, dim 128, takes 344 to 350 us by card (0.8 PFLOP/s); VALU busy 51 % and the matrix pipes
//     34 % of them, with four waves to a SIMD; waves wait 44 % of their cycles, most of that for products that follow each other and for LDS (300 us with no rows brought).
//     Fewer waves with more each were slower: 64 tokens to a wave 440 to 500 us, and with the products of one half of them beside the exponentials of the other,
//     scheduled by hand, 445 (two waves to a SIMD) and 610 (one); stages of 64 rows, four in flight, 380; neighbouring stretches on one XCD 367;
//     reads of LDS two, four or eight products ahead 349, 384 and 428 (128 registers do not hold them).
//
// Work is cut on the device, from the descriptors, into equal stretches: of units of 16 or 32 tokens of all sequences and heads, a stretch to a wave or a
// block; of steps (128 packed rows by 256 tokens) where rows are many, a stretch to a block.  A token's sum belongs to one wave, or is joined from the
// stretches that its tokens' steps fall into, in their order, by the block that ends the last: there are no atomic sums, and a batch's result is always the same bits.
#include "attention_tile.h"

namespace moe {
namespace {

constexpr int kSeqs = 256;             // sequences that are planned at a time, a thread each
constexpr int kFewRows = 16;           // packed rows of a sequence up to which they stay in registers
constexpr int kMinSteps = 2;           // of a stretch, where there are too few for all blocks (512 rows in groups of 8, us, 1 / 2 / 4: 25.8 / 26.1 / 32.7)

__device__ __forceinline__ int token_of(const WeightArgs& a, int r) { return a.G == 1 ? r : (int)divided((uint32_t)r, (uint32_t)a.G, a.g_magic); }

struct WeightSeq {
    int row0, n, p0, held;             // p0: the position of the first row; held: 0 where no score changes
    int lo;                            // the first token whose score changes
    // pieces of tok tokens (a power of two), from multiples of it
    __device__ __forceinline__ int units(int tok) const { return held > 0 ? (held - (lo & ~(tok - 1)) + tok - 1) / tok : 0; }
};
__device__ __forceinline__ WeightSeq seq_of(const WeightArgs& a, int s)
{
    WeightSeq q;
    q.row0 = a.c.off[s];
    const int hi = a.c.off[s + 1], kv = a.c.lens[s] > 0 ? a.c.lens[s] : 0;
    q.n = q.row0 < 0 || hi < q.row0 || hi > a.c.T ? 0 : hi - q.row0;
    q.held = q.n > 0 ? held_of(a.c, kv) : 0;
    q.p0 = kv - q.n;
    const int first = q.p0 - a.window + 1;
    q.lo = a.window > 0 && a.decay == 1.0f && first > 0 ? first : 0;      // (what no row sees stays as it is)
    if (q.lo >= q.held) q.held = 0;
    return q;
}

// The index of a token's score, -1 where it is not there.
__device__ __forceinline__ int64_t place_of(const WeightArgs& a, const WeightSeq& q, int seq, int h, int j)
{
    const int id = j >= q.lo && j < q.held ? a.c.table[(int64_t)seq * a.c.max_pages + (j >> a.c.page_shift)] : -1;
    return id < 0 || id >= a.c.n_pages ? -1 : page_row(id, a.c.Hk, h, a.c.page_shift, j & ((1 << a.c.page_shift) - 1));
}

// A row's lse as a power of two; infinity where the row adds nothing.
__device__ __forceinline__ float lse2_of(float lse) { return lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2e; }

__device__ __forceinline__ void store_score(const WeightArgs& a, const WeightSeq& q, int64_t at, int j, float w)
{
    if (j < q.p0 && a.decay != 0.0f) w += a.decay * a.scores[at];
    a.scores[at] = w;
}

// A value that what follows from it is not computed ahead of: the loops over stretches would keep all of that in registers.
__device__ __forceinline__ int here(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// The sum over the lane's row of sixteen.
__device__ __forceinline__ float over_sixteen(float v)
{
    auto turn = [&](auto ctrl) {
        v += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    using std::integral_constant;
    turn(integral_constant<int, 0x128>{});      // from 8, 4, 2 and 1 lanes around the sixteen
    turn(integral_constant<int, 0x124>{});
    turn(integral_constant<int, 0x122>{});
    turn(integral_constant<int, 0x121>{});
    return v;
}

// ---- few rows ----
// NJ: 16-token subtiles of a step, as the registers allow.
template <typename T, bool FP8, int DP, int NJ> struct FewWeights {
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int TOK = NJ * 16;
    static constexpr int ESZ = FP8 ? 1 : (int)sizeof(T);
    static constexpr int KC = DP / (F32 ? 16 : (FP8 ? 64 : 32));   // key loads per subtile
    static constexpr int KDIM = F32 ? 4 : (FP8 ? 16 : 8);          // dimensions of such a load
    static constexpr int KDW = KDIM * ESZ / 4;

    struct Queries {
        bf16x8_t b[F32 ? 1 : DP / 32];
        float f[F32 ? DP / 16 : 1][4];
        float lse2;
        int see_lo, see_hi;
    };
    static __device__ __forceinline__ Queries queries_of(const WeightArgs& a, const WeightSeq& q, int h, int r)
    {
        Queries Q;
        const int g = lane_id() >> 4, D = a.c.D;
        const bool there = r < q.n * a.G;
        const int tok = there ? token_of(a, r) : 0, head = h * a.G + (there ? r - tok * a.G : 0);
        const int64_t row = q.row0 + tok;
        const T* src = static_cast<const T*>(a.q) + row * a.ldq + (int64_t)head * D;
        Q.lse2 = lse2_of(a.lse[row * a.Hq + head]);
        const int p = q.p0 + tok;
        Q.see_hi = !there || Q.lse2 == __builtin_inff() ? 0 : a.causal ? p + 1 : 0x7fffffff;
        Q.see_lo = a.window > 0 ? p - a.window + 1 : 0;
        if constexpr (F32) {
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) {
                const int d = c * 16 + g * 4;
                const float4 v = *reinterpret_cast<const float4*>(src + (d < D ? d : 0));
                const bool in = d < D;
                Q.f[c][0] = in ? v.x : 0; Q.f[c][1] = in ? v.y : 0; Q.f[c][2] = in ? v.z : 0; Q.f[c][3] = in ? v.w : 0;
            }
        } else {
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) {
                const int d = FP8 ? (c / 2) * 64 + g * 16 + (c % 2) * 8 : c * 32 + g * 8;
                uint4 v = *reinterpret_cast<const uint4*>(src + (d < D ? d : 0));
                if (d >= D) v = make_uint4(0, 0, 0, 0);
                Q.b[c] = __builtin_bit_cast(bf16x8_t, v);
            }
        }
        return Q;
    }

    // Tokens [begin, end) of a sequence and head, begin a multiple of TOK; a wave's.
    static __device__ __forceinline__ void run(const WeightArgs& a, const WeightSeq& q, int seq, int h, int begin, int end)
    {
        const int lane = here(lane_id()), n = lane & 15, g = lane >> 4, D = a.c.D, shift = a.c.page_shift;
        Entries pages;
        pages.hold(a.c, seq, begin >> shift, end);
        const int rows = q.n * a.G;
        Queries Q = queries_of(a, q, h, n);

        auto page_of = [&](int t) { return __shfl(pages.id, (t >> shift) - pages.base); };
        auto slot_of = [&](int id, int t) { return page_row(id < 0 ? 0 : id, a.c.Hk, h, shift, t & ((1 << shift) - 1)); };
        // a step's loads: keys of token 16 j + n; the score that this lane will store, of token 16 (n / 4) + 4 g + n % 4
        struct Step {
            uint32_t k[NJ][KC][KDW];
            uint32_t scale[NJ];
            int64_t at;
            float old;
        };
        const int mine = (n >> 2) * 16 + 4 * g + (n & 3);
        auto load = [&](int t) {
            Step x;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int tok = t + j * 16 + n;
                const int64_t row = slot_of(page_of(tok), tok);
                const char* p = a.c.k + row * D * ESZ;
#pragma unroll
                for (int c = 0; c < KC; ++c) {
                    const int d = c * (4 * KDIM) + g * KDIM;
                    load_dwords(p + (d < D ? d : 0) * ESZ, x.k[j][c]);
                }
                if constexpr (FP8) x.scale[j] = a.c.ks[row];
            }
            const int tok = t + mine, id = page_of(n < 4 * NJ ? tok : t);
            x.at = n < 4 * NJ && id >= 0 && tok >= q.lo && tok < end ? slot_of(id, tok) : -1;
            x.old = 0;
            if (x.at >= 0 && tok < q.p0 && a.decay != 0.0f) x.old = a.scores[x.at];
            return x;
        };
        Step x = load(begin);
        for (int t = begin; t < end; t += TOK) {
            const bool more = t + TOK < end;
            if (more && ((t + 2 * TOK - 1) >> shift) - pages.base >= 64) pages.hold(a.c, seq, (t + TOK) >> shift, end);
            Step next;
            if (more) next = load(t + TOK);
            // the keys as the first product's operand
            bf16x8_t kb[F32 ? 1 : NJ][F32 ? 1 : DP / 32];
            float kf[F32 ? DP / 16 : 1][4];
            static_assert(!F32 || NJ == 1, "one subtile's keys");
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                float sc = 1.0f;
                if constexpr (FP8) sc = scale_of(x.scale[j]);
#pragma unroll
                for (int c = 0; c < KC; ++c) {
                    // (past the dimension the keys are zeros, like the queries: an infinity times zero would be NaN)
                    const bool in = c * (4 * KDIM) + g * KDIM < D;
                    uint32_t w[KDW];
#pragma unroll
                    for (int i = 0; i < KDW; ++i) w[i] = in ? x.k[j][c][i] : 0;
                    if constexpr (F32 && FP8) {
                        const hw_float2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[0], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[0], true);
                        kf[c][0] = lo[0] * sc; kf[c][1] = lo[1] * sc; kf[c][2] = hi[0] * sc; kf[c][3] = hi[1] * sc;
                    } else if constexpr (F32) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) kf[c][i] = __uint_as_float(w[i]);
                    } else if constexpr (FP8) {      // exact: a code has 4 significant bits, its scale is a power of two
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], sc, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], sc, true);
                            bf16x8_t& to = kb[j][c * 2 + i / 2];
                            to[(i % 2) * 4] = lo[0]; to[(i % 2) * 4 + 1] = lo[1]; to[(i % 2) * 4 + 2] = hi[0]; to[(i % 2) * 4 + 3] = hi[1];
                        }
                    } else {
                        kb[j][c] = __builtin_bit_cast(bf16x8_t, x.k[j][c]);
                        if (!in) kb[j][c] = bf16x8_t{};
                    }
                }
            }
            float sum[NJ][4] = {};
            for (int r0 = 0;;) {
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    float4_t s = float4_t{0, 0, 0, 0};
                    if constexpr (F32) {
#pragma unroll
                        for (int c = 0; c < DP / 16; ++c)
#pragma unroll
                            for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[c][i], Q.f[c][i], s, 0, 0, 0);
                    } else {
#pragma unroll
                        for (int c = 0; c < DP / 32; ++c) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb[j][c], Q.b[c], s, 0, 0, 0);
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int tok = t + j * 16 + 4 * g + r;
                        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.scale2, -Q.lse2));
                        sum[j][r] += ((tok < Q.see_hi) & (tok >= Q.see_lo)) ? w : 0.0f;
                    }
                }
                r0 += 16;
                if (r0 >= rows) break;      // (more than 16 rows: in batches of few rows alone, and rare)
                Q = queries_of(a, q, h, r0 + n);
            }
            if (rows > 16) Q = queries_of(a, q, h, n);
            // over the sixteen columns; lane n keeps the sum of its token
            float w = 0;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float v = over_sixteen(sum[j][r]);
                    w = n == j * 4 + r ? v : w;
                }
            if (x.at >= 0) a.scores[x.at] = __builtin_fmaf(a.decay, x.old, w);
            if (more) x = next;
        }
    }
};

// ---- many rows ----
// A dword to a lane, straight into LDS, one after the other.
__device__ __forceinline__ void load_lds_dword(uint32_t off, const char* base, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory");
}

// The steps of a sequence and head: tiles of TOK tokens, of each of which the rows that see it are taken ROWS at a time.  Tiles start at the
// position of the first row, or a whole number of tiles from it, so that the rows a causal mask leaves out are whole steps.
struct Steps {
    int first, end;                    // tiles
    int t0;                            // the tile that starts at p0
    int total;                         // steps that hold all rows
    int less;                          // by which each tile from t0 on has its rows start later (causal)
    int each;                          // steps of a tile, where they are the same for all; 0: all rows from the first that sees it
};
// EXACT: the heads are DP wide, no less.  ROWS: what 64 KB of LDS hold in two slots at dim 128, so that two blocks share a unit.
template <typename T, bool FP8, int DP, bool EXACT> struct ManyWeights {
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int WAVES = 8, WTOK = 32, TOK = WAVES * WTOK;         // tokens of a wave, of a block
    static constexpr int ROWS = F32 ? 64 : 128, PARTS = ROWS / 32;         // rows of a stage
    static constexpr int CD = F32 ? 8 : 16, KC = DP / CD, LD = CD / 2;      // dimensions of a step of the product, steps, dimensions of a lane in it
    static constexpr int ROWB = DP * (int)sizeof(T), CH = ROWB / 16;        // bytes of a row in LDS, its 16-byte chunks
    static constexpr int STAGE = ROWS * ROWB;
    static constexpr int LOADS = STAGE / (WAVES * 1024), AT = 64 / CH;                // of a wave for a stage, 1 KB each, and the rows of one
    static constexpr size_t LDS = 2 * (STAGE + ROWS * 4) + TOK * 4 + 16;    // rows and their lse, a tile's sums, a flag

    // Place of chunk 0 of row r: distinct for the rows that one read touches.
    static __device__ __forceinline__ int swz(int r)
    {
        if constexpr (ROWB == 128) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
        else return ((r & 3) << 2) | ((r >> 2) & 3);
    }

    static __device__ __forceinline__ Steps steps_of(const WeightArgs& a, const WeightSeq& q)
    {
        Steps s{0, 0, 0, 0, 0, 0};
        if (q.held == 0) return s;
        s.total = (int)(((int64_t)q.n * a.G + ROWS - 1) / ROWS);
        s.t0 = q.p0 > 0 ? (int)(((int64_t)q.p0 + TOK - 1) / TOK) : 0;
        const int64_t start = q.p0 - (int64_t)s.t0 * TOK;      // of tile 0: at most 0
        s.end = (int)((q.held - start + TOK - 1) / TOK);
        s.first = (int)((q.lo - start) / TOK);
        s.less = a.causal ? TOK / ROWS * a.G : 0;
        const int64_t band = a.causal && a.window > 0 ? (((int64_t)TOK + a.window) * a.G + ROWS - 1) / ROWS + 1 : s.total;
        s.each = !a.causal || band < s.total ? (int)band : 0;
        return s;
    }
    // steps of the tiles before t
    static __device__ __forceinline__ int64_t before(const Steps& s, int t)
    {
        if (s.each > 0) return (int64_t)(t - s.first) * s.each;
        const int64_t m = t > s.t0 ? t - (s.first > s.t0 ? s.first : s.t0) : 0, skip = s.first > s.t0 ? s.first - s.t0 : 0;
        const int64_t whole = (t < s.t0 ? t : s.t0) - s.first;
        return (whole > 0 ? whole * s.total : 0) + m * s.total - s.less * (m * (m - 1) / 2 + m * skip);
    }

    typedef __attribute__((address_space(3))) uint32x4_t lds_chunk_t;
    struct Keys {
        bf16x8_t b[F32 ? 1 : KC];
        float f[F32 ? KC : 1][4];
    };
    static __device__ __forceinline__ void load_keys(const WeightArgs& a, int64_t row, int half, Keys& K)
    {
        const int D = EXACT ? DP : a.c.D;
        float sc = 1.0f;
        if constexpr (FP8) sc = scale_of(a.c.ks[row]);
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            const int d = c * CD + half * LD;
            const char* p = a.c.k + (row * D + (d < D ? d : 0)) * (FP8 ? 1 : (int)sizeof(T));
            if constexpr (F32) {
                float4 v;
                if constexpr (FP8) {
                    const int u = *reinterpret_cast<const int*>(p);
                    const hw_float2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8(u, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(u, true);
                    v = make_float4(lo[0] * sc, lo[1] * sc, hi[0] * sc, hi[1] * sc);
                } else {
                    v = *reinterpret_cast<const float4*>(p);
                }
                K.f[c][0] = v.x; K.f[c][1] = v.y; K.f[c][2] = v.z; K.f[c][3] = v.w;
            } else if constexpr (FP8) {
                const uint2 u = *reinterpret_cast<const uint2*>(p);
                const uint32_t w[2] = {u.x, u.y};
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], sc, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], sc, true);
                    K.b[c][4 * i] = lo[0]; K.b[c][4 * i + 1] = lo[1]; K.b[c][4 * i + 2] = hi[0]; K.b[c][4 * i + 3] = hi[1];
                }
            } else {
                K.b[c] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4*>(p));
            }
        }
    }

    // What a block's threads need of a sequence and head to bring its rows into LDS and to take them against keys.
    struct Rows {
        const WeightArgs& a;
        const WeightSeq& q;
        int h, rows, tid, lane, n, half, wave, D;
        uint32_t lds0;
        float* lse;
        bool even;                                       // rows of a load are of one token, or of whole tokens, and the stages begin with one
        uint32_t lane_off, lane_chunk, lane_lse;         // then: where a lane's row and chunk are in a load, and its lse in a stage

        __device__ __forceinline__ Rows(const WeightArgs& a_, const WeightSeq& q_, int h_, char* smem) : a(a_), q(q_), h(h_)
        {
            tid = here(threadIdx.x);
            lane = tid & 63;
            n = lane & 31;
            half = lane >> 5;
            wave = __builtin_amdgcn_readfirstlane(tid >> 6);
            D = EXACT ? DP : a.c.D;
            rows = q.n * a.G;
            lds0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_address(smem));
            lse = reinterpret_cast<float*>(smem + 2 * STAGE);
            const int l = lane / CH;
            even = (a.G % AT == 0 || AT % a.G == 0) && ROWS % a.G == 0;
            lane_off = (uint32_t)(a.G % AT == 0 ? l * rowb() : token_of(a, l) * stride() + (l - token_of(a, l) * a.G) * rowb());
            lane_chunk = (uint32_t)(((lane % CH) ^ swz(l)) * 16);
            const int lr = wave * PER + lane, tok = token_of(a, lr);
            lane_lse = (uint32_t)(tok * a.Hq + lr - tok * a.G) * 4;
        }
        static constexpr int PER = ROWS / WAVES;         // rows of a wave's lse
        __device__ __forceinline__ int rowb() const { return D * (int)sizeof(T); }
        __device__ __forceinline__ int stride() const { return (int)a.ldq * (int)sizeof(T); }

        // Rows `first` on into a slot, straight into LDS, chunk c of row r to place c ^ swz(r).  A load has AT of them: where they are of one token, or of
        // whole tokens, only its address goes on from load to load; else, and where there are no more rows (the last one stands for them), every lane
        // finds its own.  (Rows of a load lie within 2^31 bytes: the launch sees to it.)
        __device__ __forceinline__ void fetch(int first, int slot) const
        {
            const T* const heads = static_cast<const T*>(a.q) + (int64_t)h * a.G * D;
            const uint32_t lse_to = lds0 + 2 * STAGE + (slot * ROWS + wave * PER) * 4;
            // (chunks past the dimension: no product reads them)
            auto inside = [&](uint32_t chunk) { return EXACT || (int)chunk < rowb() ? chunk : 0; };
            if (even && first + ROWS <= rows) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) {
                    const int lr = (wave * LOADS + i) * AT, tok = token_of(a, first + lr);
                    const char* base = reinterpret_cast<const char*>(heads + (int64_t)(q.row0 + tok) * a.ldq) + (first + lr - tok * a.G) * rowb();
                    // (the bits of a load's row in lr and those of the lane's are others, and swz takes each to a place of its own)
                    const uint32_t off[1] = {lane_off + inside(lane_chunk ^ (uint32_t)(swz(lr) * 16))};
                    load_lds_group(off, base, lds0 + slot * STAGE + lr * ROWB);
                }
                if (lane < PER)
                    load_lds_dword(lane_lse, reinterpret_cast<const char*>(a.lse + (int64_t)(q.row0 + token_of(a, first)) * a.Hq + h * a.G), lse_to);
                return;
            }
#pragma unroll 1
            for (int i = 0; i < LOADS; ++i) {
                const int lr = (wave * LOADS + i) * AT, r0 = first + lr < rows ? first + lr : rows - 1, tok0 = token_of(a, r0);
                const int r = first + lr + lane / CH < rows ? first + lr + lane / CH : rows - 1, tok = token_of(a, r);
                const char* base = reinterpret_cast<const char*>(heads + (int64_t)(q.row0 + tok0) * a.ldq);
                const uint32_t off[1] = {(uint32_t)((tok - tok0) * stride() + (r - tok * a.G) * rowb()) + inside(lane_chunk ^ (uint32_t)(swz(lr) * 16))};
                load_lds_group(off, base, lds0 + slot * STAGE + lr * ROWB);
            }
            if (lane < PER) {
                const int r = first + wave * PER + lane, rr = r < rows ? r : rows - 1, tok = token_of(a, rr), tok0 = token_of(a, first);
                load_lds_dword((uint32_t)((tok - tok0) * a.Hq + rr - tok * a.G) * 4, reinterpret_cast<const char*>(a.lse + (int64_t)(q.row0 + tok0) * a.Hq + h * a.G),
                               lse_to);
            }
        }

        // 32 rows of a slot with the wave's tokens
        __device__ __forceinline__ float16_t product(const Keys& K, int slot, int part) const
        {
            const uint32_t at = lds0 + slot * STAGE + (part * 32 + n) * ROWB + ((half ^ swz(n)) * 16);
            float16_t x = float16_t{};
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                if (!EXACT && c * CD >= D) break;
                const uint4 v = __builtin_bit_cast(uint4, *(const lds_chunk_t*)(uintptr_t)(at ^ (uint32_t)(c * 32)));
                if constexpr (F32) {
                    const float f[4] = {__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w)};
#pragma unroll
                    for (int i = 0; i < 4; ++i) x = __builtin_amdgcn_mfma_f32_32x32x2f32(K.f[c][i], f[i], x, 0, 0, 0);
                } else {
                    x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(K.b[c], __builtin_bit_cast(bf16x8_t, v), x, 0, 0, 0);
                }
            }
            return x;
        }

        // Adds the weights of a slot's rows, r0 and the ROWS - 1 after it, to the sums of tokens j0 .. j0 + 31.
        __device__ __forceinline__ void add(const Keys& K, int slot, int r0, int j0, float (&acc)[16]) const
        {
            const float* const l = lse + slot * ROWS;
            const int j1 = j0 + WTOK - 1;
            const int p_first = q.p0 + token_of(a, r0), r_last = r0 + ROWS <= rows ? r0 + ROWS - 1 : rows - 1, p_last = q.p0 + token_of(a, r_last);
            if (a.causal && p_last < j0) return;                                   // (no row sees a token of the wave)
            bool none = false;
#pragma unroll
            for (int i = 0; i < ROWS; i += 64) none |= l[i + lane] == -__builtin_inff();
            if (r0 + ROWS <= rows && (!a.causal || p_first >= j1) && (a.window == 0 || p_last - a.window + 1 <= j0) && !__any(none)) {
                // every row sees every token of the wave
#pragma unroll 1
                for (int part = 0; part < PARTS; ++part) {
                    const float l2 = l[part * 32 + n] * kLog2e;
                    const float16_t x = product(K, slot, part);
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[i] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale2, -l2));
                }
                return;
            }
#pragma unroll 1
            for (int part = 0; part < PARTS; ++part) {
                const int first = r0 + part * 32;
                if (first >= rows) break;
                const int last = first + 31 < rows ? first + 31 : rows - 1;
                if ((a.causal && q.p0 + token_of(a, last) < j0) || (a.window > 0 && q.p0 + token_of(a, first) - a.window + 1 > j1)) continue;
                const int r = first + n, p = q.p0 + token_of(a, r < rows ? r : rows - 1);
                const float raw = l[part * 32 + n], l2 = raw * kLog2e;
                const int see_hi = raw == -__builtin_inff() || r >= rows ? j0 : a.causal ? p + 1 : 0x7fffffff, see_lo = a.window > 0 ? p - a.window + 1 : -0x7fffffff;
                const float16_t x = product(K, slot, part);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = j0 + (i / 4) * 8 + 4 * half + i % 4;
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale2, -l2));
                    acc[i] += ((j < see_hi) & (j >= see_lo)) ? w : 0.0f;
                }
            }
        }

        // Sums over the 32 columns: in lanes n < 16, that of token (n / 4) * 8 + 4 half + n % 4.
        __device__ __forceinline__ float total(const float (&acc)[16]) const
        {
            float mine = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float v = over_sixteen(acc[i]);
                mine = (n & 15) == i ? v : mine;
            }
            const auto other = __builtin_amdgcn_permlane16_swap(__float_as_uint(mine), __float_as_uint(mine), false, false);
            return __uint_as_float(other[0]) + __uint_as_float(other[1]);
        }
        __device__ __forceinline__ int token() const { return (n / 4) * 8 + 4 * half + n % 4; }
    };

    // Steps [x0, x1) of a tile's `count`, as piece `piece` of `pieces`; ticket: of the tile, and where piece 0 leaves its sums.
    static __device__ __forceinline__ void run(const WeightArgs& a, const WeightSeq& q, const Steps& st, int seq, int h, int tile, int x0, int x1, int piece,
                                               int pieces, int ticket, char* smem)
    {
        const Rows R(a, q, h, smem);
        float* const sums = R.lse + 2 * ROWS;
        int32_t* const flag = reinterpret_cast<int32_t*>(sums + TOK);
        const int start = (int)(q.p0 + ((int64_t)tile - st.t0) * TOK);         // (from -TOK on)
        const int j0 = start + R.wave * WTOK;
        const int skip = tile > st.t0 ? (tile - st.t0) * st.less : 0;          // steps whose rows do not see the tile
        int r0 = (int64_t)(skip + x0) * ROWS < R.rows ? (skip + x0) * ROWS : R.rows;
        const int r1 = (int64_t)(skip + x1) * ROWS < R.rows ? (skip + x1) * ROWS : R.rows;
        if (r0 < r1) R.fetch(r0, 0);
        Keys K;
        const int64_t row = place_of(a, q, seq, h, j0 + R.n);
        load_keys(a, row < 0 ? 0 : row, R.half, K);      // (a token that is not there: some row, its sum is not stored)
        // (the compiler counts the loads it knows: waited for here, those of the keys are not waited for in the loop, where the next rows' are on the way)
        __builtin_amdgcn_s_waitcnt(0x0f70);
        float acc[16] = {};
        int slot = 0;
        for (; r0 < r1; r0 += ROWS, slot ^= 1) {
            wait_vmcnt<0>();
            block_barrier();
            if (r0 + ROWS < r1) R.fetch(r0 + ROWS, slot ^ 1);
            if (j0 < q.held) R.add(K, slot, r0, j0, acc);
        }
        const float mine = R.total(acc);
        if (R.n < 16) sums[R.wave * WTOK + R.token()] = mine;
        __syncthreads();
        const int tid = R.tid, j = start + tid;
        float w = tid < TOK ? sums[tid] : 0.0f;
        if (pieces > 1) {
            const int own = piece == 0 ? 2 * ticket + 1 : 2 * (ticket + piece);
            if (tid < TOK) store_shared(a.part + (int64_t)own * TOK + tid, w);
            if (!last_to_arrive(a.tickets + ticket, (uint32_t)pieces, flag)) return;
            if (tid < TOK) {
                w = load_shared(a.part + (int64_t)(2 * ticket + 1) * TOK + tid);
#pragma unroll 4
                for (int p = 1; p < pieces; ++p) w += load_shared(a.part + (int64_t)(2 * (ticket + p)) * TOK + tid);
            }
        }
        if (tid < TOK) {
            const int64_t at = place_of(a, q, seq, h, j);
            if (at >= 0) store_score(a, q, at, j, w);
        }
    }

    // ---- sequences whose rows fit both slots: brought there once, they meet all tokens of a stretch; every wave for itself ----
    static __device__ __forceinline__ bool fit(const WeightArgs& a, const WeightSeq& q) { return (int64_t)q.n * a.G <= 2 * ROWS; }
    // Tokens [begin, end) of a sequence and head, begin a multiple of 32.
    static __device__ __forceinline__ void run_held(const WeightArgs& a, const WeightSeq& q, int seq, int h, int begin, int end, char* smem)
    {
        const Rows R(a, q, h, smem);
        R.fetch(0, 0);
        if (R.rows > ROWS) R.fetch(ROWS, 1);
        Entries pages;
        const int shift = a.c.page_shift, mask = (1 << shift) - 1;
        auto keys_at = [&](int j0) {
            const int j = j0 + R.n, id = __shfl(pages.id, (j >> shift) - pages.base);
            return id < 0 ? (int64_t)0 : page_row(id, a.c.Hk, h, shift, j & mask);
        };
        const int first = begin + R.wave * WTOK;
        if (first < end) pages.hold(a.c, seq, first >> shift, end);
        wait_vmcnt<0>();
        block_barrier();
        for (int j0 = first; j0 < end; j0 += TOK) {
            if (((j0 + WTOK - 1) >> shift) - pages.base >= 64) pages.hold(a.c, seq, j0 >> shift, end);
            Keys K;
            load_keys(a, keys_at(j0), R.half, K);
            // (the score's place and what it was, on the way beside the keys)
            const int j = j0 + R.token(), id = __shfl(pages.id, ((R.n < 16 ? j : j0) >> shift) - pages.base);
            const int64_t at = R.n < 16 && id >= 0 && j >= q.lo && j < end ? page_row(id, a.c.Hk, h, shift, j & mask) : -1;
            const float old = at >= 0 && j < q.p0 && a.decay != 0.0f ? a.scores[at] : 0.0f;
            float acc[16] = {};
            for (int slot = 0; slot * ROWS < R.rows; ++slot) R.add(K, slot, slot * ROWS, j0, acc);
            const float w = R.total(acc);
            if (at >= 0) a.scores[at] = __builtin_fmaf(a.decay, old, w);
        }
    }
};

// Sums of a quantity over the sequences up to and with each, of kSeqs sequences.
struct WeightPlan {
    int64_t upto[kSeqs];
    int64_t sums[8];
};
__device__ __forceinline__ int64_t scan64(int64_t v)
{
    for (int d = 1; d < 64; d *= 2) {
        const int64_t o = __shfl_up(v, d);
        if (lane_id() >= d) v += o;
    }
    return v;
}
// Every thread of the block calls it, the first kSeqs with their sequence's value; a barrier comes between two plans that share LDS.
__device__ __forceinline__ void make_plan(WeightPlan& plan, int64_t v)
{
    const int wave = threadIdx.x >> 6;
    v = scan64(v);
    if (lane_id() == 63) plan.sums[wave] = v;
    __syncthreads();
    for (int w = 0; w < wave; ++w) v += plan.sums[w];
    if (threadIdx.x < kSeqs) plan.upto[threadIdx.x] = v;
    __syncthreads();
}
// The first sequence whose sum is above x, and the sum before it.
__device__ __forceinline__ int found_in(const WeightPlan& plan, int64_t x, int64_t& before)
{
    int lo = 0, hi = kSeqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (plan.upto[mid] > x) hi = mid;
        else lo = mid + 1;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    before = lo > 0 ? plan.upto[lo - 1] : 0;
    return lo;
}

// The stretch [x, end) of a plan of units (of tok tokens of a sequence and head): f(sequence's number in the plan, its data, head, tokens begin .. end - 1).
template <typename F> __device__ __forceinline__ void each_span(const WeightArgs& a, const WeightPlan& plan, int s0, int tok, int64_t x, int64_t end, F f)
{
    while (x < end) {
        int64_t base;
        const int i = found_in(plan, x, base);
        const WeightSeq q = seq_of(a, s0 + i);
        const int units = q.units(tok), h = (int)((x - base) / units), from = (int)(x - base - (int64_t)h * units);
        const int to = end - x < units - from ? from + (int)(end - x) : units;
        const int begin = (q.lo & ~(tok - 1)) + from * tok, stop = begin + (to - from) * tok < q.held ? begin + (to - from) * tok : q.held;
        f(s0 + i, q, h, begin, stop);
        x += to - from;
    }
}

// Sequences of up to a.few_rows packed rows.  Blocks of a unit: 64 decode rows over up to 8192 tokens, us, as here / one more: bf16 dim 128 44 / 54, 256 80 / 119;
// one fewer: FP8 128 27 / 29, fp32 128 30 / 37, two fewer: bf16 64 47 / 51.
template <typename T, bool FP8, int DP> struct FewKernel {
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int BLOCKS = DP > 128 ? 1 : DP > 64 ? (FP8 ? (F32 ? 2 : 3) : 2) : F32 ? 3 : 4;
};
template <typename T, bool FP8, int DP> __global__ __launch_bounds__(256, (FewKernel<T, FP8, DP>::BLOCKS)) void few_weights_kernel(WeightArgs a)
{
    typedef FewWeights<T, FP8, DP, sizeof(T) == 4 ? 1 : 2> Few;
    __shared__ WeightPlan plan;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    for (int s0 = 0; s0 < a.c.S; s0 += kSeqs) {
        const int s = s0 + threadIdx.x;
        int64_t units = 0;
        if (s < a.c.S) {
            const WeightSeq q = seq_of(a, s);
            if (q.n * a.G <= a.few_rows) units = (int64_t)q.units(Few::TOK) * a.c.Hk;
        }
        make_plan(plan, units);
        const int64_t all = plan.upto[kSeqs - 1], waves = (int64_t)gridDim.x * 4, me = (int64_t)blockIdx.x * 4 + wave;
        each_span(a, plan, s0, Few::TOK, me * all / waves, (me + 1) * all / waves,
                  [&](int seq, const WeightSeq& q, int h, int begin, int end) { Few::run(a, q, seq, h, begin, end); });
        __syncthreads();
    }
}

// Sequences of more packed rows than a.few_rows.  Registers kept in scratch: 7 at 128 dimensions in bf16 (FP8 pages 8), 21 at 80 to 112; fp32 16 below 64 and 81
// (FP8 pages 54) at 144 to 240.  A prompt of 2048 rows, 32 heads over 4, bf16, us: 48 dimensions 43, 64 42, 80 51, 96 52, 112 53, 128 49, 144 60, 208 66, 256 68 (FP8 the
// same within 2 %); fp32, 1024 rows: 54, 55, 53, 59, 63, 63, 78, 99, 106.
template <typename T, bool FP8, int DP, bool EXACT> struct RowsKernel {
    typedef ManyWeights<T, FP8, DP, EXACT> Many;
    static constexpr int THREADS = 64 * Many::WAVES, BLOCKS = DP > 128 || (sizeof(T) == 4 && DP > 64) ? 1 : 2;      // of a unit
    static constexpr size_t PLAN_AT = (Many::LDS + 15) / 16 * 16, LDS = PLAN_AT + 2 * sizeof(WeightPlan);
};
template <typename T, bool FP8, int DP, bool EXACT>
__global__ __launch_bounds__((RowsKernel<T, FP8, DP, EXACT>::THREADS), (RowsKernel<T, FP8, DP, EXACT>::BLOCKS * 2)) void rows_weights_kernel(WeightArgs a)
{
    typedef RowsKernel<T, FP8, DP, EXACT> K;
    typedef typename K::Many Many;
    extern __shared__ __attribute__((aligned(256))) char smem[];
    WeightPlan *const held = reinterpret_cast<WeightPlan*>(smem + K::PLAN_AT), *const many = held + 1;
    for (int s0 = 0; s0 < a.c.S; s0 += kSeqs) {
        const int s = s0 + threadIdx.x;
        int64_t units = 0, steps = 0;
        if (threadIdx.x < kSeqs && s < a.c.S) {
            const WeightSeq q = seq_of(a, s);
            if (q.n * a.G > a.few_rows) {
                if (Many::fit(a, q)) {
                    units = (int64_t)q.units(Many::WTOK) * a.c.Hk;
                } else {
                    const Steps st = Many::steps_of(a, q);
                    steps = Many::before(st, st.end) * a.c.Hk;
                }
            }
        }
        make_plan(*held, units);
        make_plan(*many, steps);
        const int chunk = s0 / kSeqs;
        const bool split = chunk < a.split_chunks;                       // (where there are no more slots, a tile is its first step's owner's)
        int64_t all = many->upto[kSeqs - 1];
        const int64_t most = (all + kMinSteps - 1) / kMinSteps;
        const int64_t blocks = most < gridDim.x ? most : gridDim.x;      // that have a stretch
        auto cut = [&](int64_t b) { return b * all / blocks; };
        if ((int64_t)blockIdx.x < blocks) {
            // the stretch that step x lies in
            auto owner = [&](int64_t x) {
                int64_t b = x * blocks / all;
                while (cut(b + 1) <= x) ++b;
                return (int)b;
            };
            const int64_t start = cut(blockIdx.x), end = cut(blockIdx.x + 1);
            int64_t x = start;
            while (x < end) {
                int64_t base;
                const int i = found_in(*many, x, base);
                const WeightSeq q = seq_of(a, s0 + i);
                const Steps st = Many::steps_of(a, q);
                const int64_t of_head = Many::before(st, st.end);
                const int h = (int)((x - base) / of_head);
                const int64_t head_base = base + h * of_head, rem = x - head_base;
                int lo = st.first, hi = st.end - 1;                      // the last tile that starts at or before rem
                while (lo < hi) {
                    const int mid = (lo + hi + 1) / 2;
                    if (Many::before(st, mid) <= rem) lo = mid;
                    else hi = mid - 1;
                }
                for (int tile = lo; tile < st.end && x < end; ++tile) {
                    const int64_t t_begin = head_base + Many::before(st, tile), t_end = head_base + Many::before(st, tile + 1);
                    const int64_t to = !split || t_end < end ? t_end : end;
                    if (split || x == t_begin) {
                        int first = (int)blockIdx.x, last = first;
                        if (split && t_begin < start) first = owner(t_begin);
                        if (split && t_end > end) last = owner(t_end - 1);
                        Many::run(a, q, st, s0 + i, h, tile, (int)(x - t_begin), (int)(to - t_begin), (int)blockIdx.x - first, last - first + 1,
                                  chunk * (int)gridDim.x + first, smem);
                        __syncthreads();
                    }
                    x = to;
                }
            }
        }
        all = held->upto[kSeqs - 1];
        each_span(a, *held, s0, Many::WTOK, blockIdx.x * all / gridDim.x, (blockIdx.x + 1) * all / gridDim.x,
                  [&](int seq, const WeightSeq& q, int h, int begin, int end) {
                      Many::run_held(a, q, seq, h, begin, end, smem);
                      __syncthreads();
                  });
        __syncthreads();
    }
}

template <typename T, bool FP8, int DP> hipError_t launch_few(const WeightArgs& a, int units, hipStream_t s)
{
    few_weights_kernel<T, FP8, DP><<<(unsigned)(units * FewKernel<T, FP8, DP>::BLOCKS), 256, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T, bool FP8, int DP, bool EXACT> hipError_t launch_rows(WeightArgs a, int units, bool clear_tickets, hipStream_t s)
{
    typedef RowsKernel<T, FP8, DP, EXACT> K;
    static bool done[kMaxDevices];
    const auto kern = rows_weights_kernel<T, FP8, DP, EXACT>;
    hipError_t e = ensure_lds_limit(kern, K::LDS, done);
    if (e != hipSuccess) return e;
    if (clear_tickets && (e = launch_fill_zero(a.tickets, kPartUnits, s)) != hipSuccess) return e;
    int grid = units * K::BLOCKS;
    if (grid > kPartUnits) grid = kPartUnits;      // (a ticket to a stretch)
    a.split_chunks = (int)((int64_t)kPartUnits * 16 * a.c.D / (2 * K::Many::TOK) / grid);      // two slots of partial sums to a stretch
    if (a.split_chunks > kPartUnits / grid) a.split_chunks = kPartUnits / grid;
    kern<<<(unsigned)grid, K::THREADS, K::LDS, s>>>(a);
    return hipGetLastError();
}

template <typename T, bool FP8, int DP> hipError_t launch_by_rows(WeightArgs a, bool& clear, hipStream_t s)
{
    int units = 0;
    hipError_t e = compute_units(&units);
    if (e != hipSuccess) return e;
    a.g_magic = a.G > 1 ? (uint32_t)((((uint64_t)1 << 32) + a.G - 1) / a.G) : 0;
    // How rows spread over the sequences only the device knows.  A batch of decode or drafted rows alone, by the rule of the attention's launch, is one of few
    // rows throughout; one that is mostly such takes two launches, one for its sequences of few rows and one for the rest; in any other the kernel of many rows
    // takes all.  A prompt's 512 rows over 8192 tokens among decode rows, dim 128, us, one launch / two, decode rows over up to 4096 tokens and, in brackets, 300:
    //   groups of 8, 4 key/value heads: 31 rows bf16 75 / 82; 63 FP8 83 / 84; behind the line 95 bf16 99 / 106 (70 / 72), FP8 94 / 90 (70 / 73), fp32 392 / 376;
    //     255 bf16 160 / 166 (82 / 77), FP8 143 / 125 (83 / 76), fp32 528 / 488
    //   groups of 4, 8 heads: 40 bf16 90 / 96 (68 / 66), FP8 87 / 81 (67 / 66), fp32 386 / 373; 255 bf16 262 / 255 (106 / 79), FP8 221 / 174 (110 / 75), fp32 762 / 670
    //   groups of one, 8 heads: 10 bf16 37 / 41 (31 / 33), FP8 39 / 39 (32 / 35), fp32 117 / 116; 255 bf16 235 / 223 (74 / 46), FP8 192 / 144 (79 / 44), fp32 547 / 452
    // (What two launches lose near the line, in bf16 above all, is up to 7 us; what they save behind it grows with the decode rows, the more the fewer heads a group has.)
    constexpr int kMostRows = 384;
    const int64_t rows = a.c.T, seqs = a.c.S, most = rows < seqs ? rows : rows - seqs + 1;
    if (rows * a.G <= kFewRows * seqs && most * a.G <= kMostRows) {
        a.few_rows = 0x7fffffff;
        clear = false;
        return launch_few<T, FP8, DP>(a, units, s);
    }
    a.few_rows = rows * a.G <= 4 * kFewRows * seqs ? kFewRows : 0;
    if (a.few_rows > 0 && (e = launch_few<T, FP8, DP>(a, units, s)) != hipSuccess) return e;
    return a.c.D == DP ? launch_rows<T, FP8, DP, true>(a, units, clear, s) : launch_rows<T, FP8, DP, false>(a, units, clear, s);
}

template <typename T, bool FP8> hipError_t launch_by_dim(const WeightArgs& a, bool& clear, hipStream_t s)
{
    if (a.c.D <= 64) return launch_by_rows<T, FP8, 64>(a, clear, s);
    if (a.c.D <= 128) return launch_by_rows<T, FP8, 128>(a, clear, s);
    return launch_by_rows<T, FP8, 256>(a, clear, s);
}

}  // namespace

hipError_t launch_kv_weights(int dtype, bool fp8, const WeightArgs& a, bool& clear, hipStream_t s)
{
    if (dtype == MOE_BF16) return fp8 ? launch_by_dim<bf16_t, true>(a, clear, s) : launch_by_dim<bf16_t, false>(a, clear, s);
    return fp8 ? launch_by_dim<float, true>(a, clear, s) : launch_by_dim<float, false>(a, clear, s);
}

}  // namespace moe
