#pragma once
#include "attention_plan.h"
#include "ffn_tile.h"

namespace moe {
namespace {

// ----------------------------------------------------------------------------------------------------------------
// The kernel for many rows (bf16): tiles of 128 packed rows, 32 to a wave, over steps of 64 tokens whose keys and values the
// block stages in LDS, two steps in turn.
//
// Both products are transposed as in attention_few.h, here with 32 x 32 matrix instructions: a lane holds column q = lane % 32 of
// the scores and of the output, so maxima, sums and scales are lane-local but for one exchange between the wave's halves, and the
// exponentials are the second product's operand where they stand.  Its other operand, V transposed, comes out of LDS through
// the transposing reads (a lane gets one dimension of four tokens), in the token order that the exponentials happen to have.
// A row of 256 bytes would put the same dimensions of every token on the same banks; its 16-byte chunks are permuted, chunk c of
// token t in place c ^ swz(t), so that both kinds of read touch every bank equally.
//
// Why 128 rows and four waves: a step's 32 KB of operands are read from LDS by every wave for its 32 rows, 128 bytes a cycle if the matrix
// pipes never paused, and two such blocks share a unit, each with its own barrier, so that one's exponentials run beside the other's
// products.  What bounds it at dim 128: the matrix pipes at the clock that they leave (2.0 GHz), busy 45 % of a causal prompt of 8192 tokens and 32
// heads (573 us with 128 decode rows, 0.96 PFLOP/s), half of all steps' issue being vector instructions.  8192 rows to 8192 tokens, no
// mask, 32 heads: dim 128 1043 us (1.05 PFLOP/s), FP8 pages 1139; dim 64 628 (0.88: as many exponentials for half the products), FP8 666; 4096 to 4096,
// 16 heads, dim 256, one block to a unit: 420 (0.65).
// ----------------------------------------------------------------------------------------------------------------
constexpr int kManyRows = 128;

// N direct-to-LDS loads of a wave, 1 KB after the other in LDS and, but for what the offsets make good, in memory (the
// instruction's offset counts in both): M0 is written once for all of them.
constexpr uint32_t kGroupBias = 3 * 1024;    // keeps the 32-bit offsets from falling below zero
template <int N> __device__ __forceinline__ void load_lds_group(const uint32_t (&off)[N], const char* base, uint32_t lds)
{
    if constexpr (N == 1)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off[0]), "s"(base), "s"(lds) : "memory");
    else if constexpr (N == 2)
        asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2\n\tglobal_load_lds_dwordx4 %1, %2 offset:1024" ::"v"(off[0]),
                     "v"(off[1]), "s"(base), "s"(lds) : "memory");
    else
        asm volatile("s_mov_b32 m0, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %4\n\tglobal_load_lds_dwordx4 %1, %4 offset:1024\n\t"
                     "global_load_lds_dwordx4 %2, %4 offset:2048\n\tglobal_load_lds_dwordx4 %3, %4 offset:%6" ::"v"(off[0]), "v"(off[1]),
                     "v"(off[2]), "v"(off[3]), "s"(base), "s"(lds), "n"(kGroupBias) : "memory");
}

template <bool FP8, int DP, bool EXACT, bool TREE> struct Many {
    static constexpr int TOK = 64;
    static constexpr int ROWB = DP * 2;              // bytes of a token's row in LDS
    static constexpr int CH = DP / 8;                // its 16-byte chunks
    static constexpr int HALF = TOK * ROWB;          // keys, then values
    static constexpr int STAGE = 2 * HALF;
    static constexpr size_t LDS = 2 * STAGE + 16;    // (and a flag)
    static constexpr int NB = DP / 32;               // output blocks of 32 dimensions
    static constexpr int LOADS = TOK * CH / 256;     // 16-byte loads of a thread for a step's keys (as many for its values)

    // place of chunk 0 of token t: distinct for the tokens that one read touches, within the chunks of 256 bytes
    static __device__ __forceinline__ int swz(int t)
    {
        if constexpr (DP == 64) return (((t >> 1) & 1) << 2) | ((t >> 2) & 3);
        else return ((t & 3) << 2) | ((t >> 2) & 3);
    }

    static __device__ __forceinline__ float swap_max(float v)
    {
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
    }
    static __device__ __forceinline__ float swap_sum(float v)
    {
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return __uint_as_float(x[0]) + __uint_as_float(x[1]);
    }

    // A step of 64 tokens; bit i of `there`: tokens t + 8 i .. t + 8 i + 7 are (pages hold whole groups of eight).
    struct Step {
        int t;
        uint32_t there;
    };

    typedef short short4_t __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) short4_t lds_short4_t;
    static __device__ __forceinline__ uint2 read_transposed(uint32_t lds)
    {
        return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t*)(uintptr_t)lds));
    }
    // Values of tokens 16 k .. 16 k + 15 in the order of the exponentials, dimensions 32 x .. 32 x + 31.
    static __device__ __forceinline__ bf16x8_t read_values(const uint32_t (&v_at)[2][NB], int k, int x)
    {
        const uint2 lo = read_transposed(v_at[0][x] + k * 16 * ROWB), hi = read_transposed(v_at[1][x] + k * 16 * ROWB);
        return __builtin_bit_cast(bf16x8_t, make_uint4(lo.x, lo.y, hi.x, hi.y));
    }
    typedef __attribute__((address_space(3))) uint32x4_t lds_chunk_t;
    static __device__ __forceinline__ bf16x8_t read_keys(uint32_t lds)
    {
        return __builtin_bit_cast(bf16x8_t, *(const lds_chunk_t*)(uintptr_t)lds);
    }

    static __device__ __forceinline__ void run(const AttnArgs& a, const Item& it, char* smem)
    {
        const Range rg = range_of<TREE>(a, it);
        if (it.sub >= rg.pieces) return;
        const int lane = lane_id(), n = lane & 31, h = lane >> 5;
        const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
        const int D = EXACT ? DP : a.c.D, shift = a.c.page_shift, Hk = a.c.Hk;
        const uint32_t lds0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_address(smem));

        auto me = row_of<TREE>(a, it, rg, rg.first + wave * 32 + n);
        bf16x8_t qf[DP / 16];
        {
            const bf16_t* src = static_cast<const bf16_t*>(a.q) + (int64_t)me.row * a.ldq + (int64_t)me.head * D;
#pragma unroll
            for (int s = 0; s < DP / 16; ++s) {
                const int d = s * 16 + h * 8;
                uint4 v = *reinterpret_cast<const uint4*>(src + (d < D ? d : 0));
                if (!me.there || d >= D) v = make_uint4(0, 0, 0, 0);
                qf[s] = __builtin_bit_cast(bf16x8_t, v);
            }
        }

        // ---- staging: a wave's share of a step are 16 tokens, two groups of eight ----
        // Per held entry of the page table, the byte offset of this head's first token in the pages (and its row, for the scales):
        // a step then takes what it needs as scalars, and no lane works out an address.
        Entries pages;
        unsigned long long held = 0;
        uint32_t byte_lo = 0, byte_hi = 0, row_lo = 0, row_hi = 0;
        auto hold = [&](int page) {
            pages.hold(a.c, it.seq, page, rg.end);
            held = __ballot(pages.id >= 0);
            const int64_t row = page_row(pages.id < 0 ? 0 : pages.id, Hk, it.head, shift, 0);
            const int64_t byte = row * (D * (FP8 ? 1 : 2));
            byte_lo = (uint32_t)byte;
            byte_hi = (uint32_t)((uint64_t)byte >> 32);
            row_lo = (uint32_t)row;
            row_hi = (uint32_t)((uint64_t)row >> 32);
        };
        auto step_at = [&](int t) {
            if (((t + TOK - 1) >> shift) - pages.base >= 64) hold(t >> shift);
            const int first = (t >> shift) - pages.base, last = ((t + TOK - 1) >> shift) - pages.base;
            Step s{t, 0xffu};
            if ((~(held >> first) << (63 - (last - first))) != 0) {
                s.there = 0;
#pragma unroll
                for (int i = 0; i < TOK / 8; ++i) s.there |= (uint32_t)((held >> (((t + 8 * i) >> shift) - pages.base)) & 1) << i;
            }
            return s;
        };
        auto lane64 = [](uint32_t lo, uint32_t hi, int i) {
            return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)lo, i) |
                             (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)hi, i) << 32);
        };
        const int mask = (1 << shift) - 1;
        // bf16: straight into LDS, 64 / CH tokens to a load; the loads of a group follow each other in LDS
        constexpr int TPL = 64 / CH, GL = LOADS / 2;
        uint32_t from[2][GL];
        if constexpr (!FP8) {
            const int tl = lane / CH, c = lane % CH;
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int i = 0; i < GL; ++i) {
                    // (chunks past the dimension: no product reads those of the keys, those of the values go to outputs that are not stored)
                    const int chunk = c ^ swz(g * 8 + i * TPL + tl);
                    from[g][i] = (uint32_t)((i * TPL + tl) * D * 2 + (chunk * 8 < D ? chunk * 16 : 0) - i * 1024) + kGroupBias;
                }
        }
        auto stage = [&](const Step& s, uint32_t base) {
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const int t = s.t + wave * 16 + g * 8;
                const int64_t off = lane64(byte_lo, byte_hi, (t >> shift) - pages.base) + (t & mask) * (D * 2) - (int)kGroupBias;
                const uint32_t to = base + (wave * 16 + g * 8) * ROWB;
                load_lds_group(from[g], a.c.k + off, to);
                load_lds_group(from[g], a.c.v + off, to + HALF);
            }
        };
        // FP8: 16 codes to a lane, through registers, widened exactly (a code has 4 significant bits, its scale is a power of two)
        constexpr int LPT = DP / 16;                   // lanes to a token
        constexpr int TPW = 64 / LPT;                  // tokens to a wave's load
        constexpr int FL = TOK / (4 * TPW);            // loads of a wave
        uint4 raw[FP8 ? FL : 1][2];
        uint32_t raw_scale[FP8 ? FL : 1][2];
        auto fetch = [&](const Step& s) {
            const int tl = lane / LPT, c = lane % LPT;
            int64_t byte[2], row[2];
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const int t = s.t + wave * 16 + g * 8, i = (t >> shift) - pages.base;
                byte[g] = lane64(byte_lo, byte_hi, i) + (t & mask) * D;
                row[g] = lane64(row_lo, row_hi, i) + (t & mask);
            }
#pragma unroll
            for (int i = 0; i < FL; ++i) {
                const int t = i * TPW + tl;            // of the wave's 16
                const bool second = TPW > 8 ? t >= 8 : i * TPW >= 8;
                const int64_t bb = second ? byte[1] : byte[0], rr = second ? row[1] : row[0];
                const uint32_t off = (uint32_t)((t & 7) * D + (c * 16 < D ? c * 16 : 0));
                raw[i][0] = *reinterpret_cast<const uint4*>(a.c.k + bb + off);
                raw[i][1] = *reinterpret_cast<const uint4*>(a.c.v + bb + off);
                raw_scale[i][0] = (a.c.ks + rr)[t & 7];
                raw_scale[i][1] = (a.c.vs + rr)[t & 7];
            }
        };
        auto widen = [&](char* base) {
            const int tl = lane / LPT, c = lane % LPT;
#pragma unroll
            for (int i = 0; i < FL; ++i) {
                const int t = wave * 16 + i * TPW + tl;
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    const float sc = scale_of(raw_scale[i][kv]);
                    const uint32_t w[4] = {raw[i][kv].x, raw[i][kv].y, raw[i][kv].z, raw[i][kv].w};
                    uint32_t o[8];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        o[2 * x] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[x], sc, false));
                        o[2 * x + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[x], sc, true));
                    }
                    char* row = base + kv * HALF + t * ROWB;
                    *reinterpret_cast<uint4*>(row + ((2 * c) ^ swz(t)) * 16) = make_uint4(o[0], o[1], o[2], o[3]);
                    *reinterpret_cast<uint4*>(row + ((2 * c + 1) ^ swz(t)) * 16) = make_uint4(o[4], o[5], o[6], o[7]);
                }
            }
        };

        // ---- operand addresses in the step's stage ----
        // keys: token 32 b + n, chunk 2 c + h
        uint32_t k_at[DP / 16];
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) k_at[c] = lds0 + n * ROWB + (((2 * c + h) ^ swz(n)) * 16);
        // values: tokens 16 k + 8 u + 4 h + (lane % 16) / 4, dimensions 32 x + 16 (lane / 16 % 2) + 4 (lane % 4): see read_transposed
        uint32_t v_at[2][NB];
        {
            const int tok = 4 * h + ((lane & 15) >> 2), chunk = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int x = 0; x < NB; ++x)
                    v_at[u][x] = lds0 + HALF + (8 * u + tok) * ROWB + (lane & 1) * 8 + (((chunk + 4 * x) ^ swz(8 * u + tok)) * 16);
        }

        float m = kLowest, l = 0;
        float16_t o[NB];
#pragma unroll
        for (int x = 0; x < NB; ++x) o[x] = float16_t{};

        Step cur{rg.begin, 0};
        if (rg.begin < rg.end) {
            hold(rg.begin >> shift);
            cur = step_at(rg.begin);
            if constexpr (FP8) {
                fetch(cur);
                widen(smem);
            } else {
                stage(cur, lds0);
            }
        }
        const bool idle = rg.first + wave * 32 >= rg.rows;           // a wave whose rows are none stages all the same
        // The compiler counts the loads it knows: without this wait it would put one for the queries into the loop, where it would
        // also wait for the loads of the step after.
        __builtin_amdgcn_s_waitcnt(0x0f70);                          // vmcnt(0)
        int at = 0;                                                  // byte offset of the step's stage
        while (cur.t < rg.end) {
            if constexpr (FP8) wait_lds_reads();
            else wait_vmcnt<0>();
            block_barrier();
            // a step whose tokens not every row sees
            const bool masked = cur.t + TOK > rg.full_hi || cur.t < rg.full_lo || cur.there != 0xffu;
            if (masked) me.sight.step(a, cur.t);
            if (masked) clean_values(cur, rg, me, v_at, lds0 + at + HALF, smem, o);
            Step next{cur.t + TOK, 0};
            const bool more = next.t < rg.end;
            if (more) {
                next = step_at(next.t);
                if constexpr (FP8) fetch(next);
                else stage(next, lds0 + (at ^ STAGE));
            }
            if (!idle) {
                float16_t s[2];
#pragma unroll
                for (int c = 0; c < DP / 16; ++c) {
                    // Past the dimension: what is staged there is no key, and an infinity of it would be NaN against a query of zeros.  Its products
                    // are left out, at 256 its chunks are made zeros (3000 rows to 3000 tokens, 32 heads, us, products of it all / left out / zeros: dim 80
                    // 95 / 88 / -, 112 94 / 89 / -, 208 273 / 381 / 280: with one wave to a SIMD nothing hides the reads of a loop in pieces).
                    if (!EXACT && DP <= 128 && c * 16 >= D) break;
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        bf16x8_t key = read_keys(k_at[c] + b * 32 * ROWB);
                        if (!EXACT && DP > 128 && c * 16 >= DP / 2 && c * 16 >= D) key = bf16x8_t{};
                        s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key, qf[c], c == 0 ? float16_t{} : s[b], 0, 0, 0);
                    }
                }
                if (masked) {
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int grp = b * 4 + r / 4, tok = cur.t + grp * 8 + 4 * h + r % 4;
                            const bool sees = (((cur.there >> grp) & 1) != 0) & me.sight.sees(tok);
                            s[b][r] = sees ? s[b][r] : -__builtin_inff();
                        }
                }
                float top = -__builtin_inff();
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[b][r]);
                top = swap_max(top) * a.scale2;                      // (the scale is positive)
                // (the reference of the exponentials follows the maximum only when that has grown by more than 8, see attention_few.h)
                // Before a row's first token there is nothing to scale but what clean_values gave it in this step, which no factor may touch:
                // zero times an infinity would be NaN.
                if (__any(top > m + 8.0f)) {
                    const float to = fmaxf(top, m), f = m == kLowest ? 1.0f : __builtin_amdgcn_exp2f(m - to);
                    m = to;
                    l *= f;
#pragma unroll
                    for (int x = 0; x < NB; ++x) o[x] *= f;
                }
                bf16x8_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t u[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k / 2][(k % 2) * 8 + 2 * i], a.scale2, -m));
                        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k / 2][(k % 2) * 8 + 2 * i + 1], a.scale2, -m));
                        l += p0;
                        l += p1;
                        u[i] = pack_bf16x2(p0, p1);      // (see Few::weights_of)
                    }
                    w[k] = __builtin_bit_cast(bf16x8_t, make_uint4(u[0], u[1], u[2], u[3]));
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int x = 0; x < NB; ++x)
                        o[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_values(v_at, k, x), w[k], o[x], 0, 0, 0);
            }
            if constexpr (FP8)
                if (more) widen(smem + (at ^ STAGE));
            const int turn = at == 0 ? STAGE : -STAGE;
            at += turn;
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) k_at[c] += turn;
#pragma unroll
            for (int x = 0; x < NB; ++x) {
                v_at[0][x] += turn;
                v_at[1][x] += turn;
            }
            cur = next;
        }

        // Results: a wave turns its 32 rows by way of LDS, so that they leave in whole rows.  Chunk c (four dimensions) of row q
        // sits in place c ^ (q % chunks).
        l = swap_sum(l);
        const Finish fin = finish_row(a, me.head, m, l);
        const float f = rg.pieces > 1 ? 1.0f : fin.factor;
        const int part = (it.slot + it.sub * it.q.units) * 16 + wave * 32;
        if (me.there && h == 0) {
            if (rg.pieces > 1) store_part_stats(a, part + n, m, l);
            else if (a.lse) a.lse[(int64_t)me.row * a.Hq + me.head] = fin.lse;
        }
        constexpr int OC = DP / 4, RPI = 64 / (OC < 64 ? OC : 64);     // chunks of a row, rows to 64 lanes
        __syncthreads();                                             // (the stages are no longer read)
        char* mine = smem + wave * 32 * DP * 4;
#pragma unroll
        for (int x = 0; x < NB; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *reinterpret_cast<float4*>(mine + n * DP * 4 + (((x * 8 + r * 2 + h) ^ (n & (OC - 1))) * 16)) =
                    make_float4(o[x][4 * r] * f, o[x][4 * r + 1] * f, o[x][4 * r + 2] * f, o[x][4 * r + 3] * f);
        __builtin_amdgcn_wave_barrier();                             // (a wave's LDS operations keep their order)
        const Parts parts = parts_of(a, D);
        const int c = lane % OC;
#pragma unroll
        for (int i = 0; i < 32 / RPI; ++i) {
            const int q = i * RPI + lane / OC;
            const float4 v = *reinterpret_cast<const float4*>(mine + q * DP * 4 + ((c ^ (q & (OC - 1))) * 16));
            const auto row = row_of<TREE>(a, it, rg, rg.first + wave * 32 + q);
            if (row.there && c * 4 < D) {
                if (rg.pieces > 1) store_part(parts, part + q, c * 4, v);
                else store_out<bf16_t>(a, row.row, row.head, D, c * 4, v);
            }
        }
        if (rg.pieces > 1) {
            __syncthreads();                                         // the flag shares the stages' memory
            join_pieces<bf16_t, DP, 8, TREE>(a, it, rg, D, reinterpret_cast<int32_t*>(smem));
        }
    }

    // The values of a step whose tokens not every row sees, made fit for the second product, where a weight of zero keeps only finite
    // values out: tokens that are not there, or that no row sees, become zeros, whatever the cache holds; where there is an infinity or NaN
    // among the others, the rows that see it get it right away, and it becomes a zero too.  Every thread of the block calls it.
    static __device__ __forceinline__ void clean_values(const Step& cur, const Range& rg, const Row<TREE>& me, const uint32_t (&v_at)[2][NB],
                                                        uint32_t values, char* smem, float16_t (&o)[NB])
    {
        int32_t* flag = reinterpret_cast<int32_t*>(smem + 2 * STAGE);
        auto mine = [&](auto f) {
            for (int i = threadIdx.x; i < TOK * CH; i += 256) {
                const int tl = i / CH;
                uint4 v = read_chunk(values + i * 16);
                if (f(v, ((cur.there >> (tl / 8)) & 1) != 0 && cur.t + tl < rg.hi)) write_chunk(values + i * 16, v);
            }
        };
        if (threadIdx.x == 0) *flag = 0;
        __syncthreads();
        mine([&](uint4& v, bool there) {
            if (!there) {
                v = make_uint4(0, 0, 0, 0);
                return true;
            }
            if (strange(v.x) | strange(v.y) | strange(v.z) | strange(v.w)) *flag = 1;
            return false;
        });
        __syncthreads();
        if (*flag == 0) return;
        give_strange_values(cur, me, v_at, o);
        __syncthreads();
        mine([&](uint4& v, bool) {
            v.x = finite_of(v.x); v.y = finite_of(v.y); v.z = finite_of(v.z); v.w = finite_of(v.w);
            return true;
        });
        __syncthreads();
    }
    static __device__ __forceinline__ void give_strange_values(const Step& cur, const Row<TREE>& me, const uint32_t (&v_at)[2][NB], float16_t (&o)[NB])
    {
        const int h = lane_id() >> 5;
#pragma unroll
        for (int x = 0; x < NB; ++x)
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {
                uint32_t seen[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    seen[i] = 0;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int grp = 2 * k + i / 2, tok = cur.t + grp * 8 + 4 * h + (i % 2) * 2 + e;
                        if (((cur.there >> grp) & 1) && me.sight.sees(tok)) seen[i] |= 0x3f80u << (16 * e);
                    }
                }
                const uint4 v = __builtin_bit_cast(uint4, read_values(v_at, k, x));
                const uint32_t vv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll 1
                for (int what = 1; what <= 3; ++what) {
                    uint32_t mark[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        mark[i] = (kind(vv[i] & 0xffffu) == what ? 0x3f80u : 0u) | (kind(vv[i] >> 16) == what ? 0x3f800000u : 0u);
                    const float16_t hits = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        __builtin_bit_cast(bf16x8_t, make_uint4(mark[0], mark[1], mark[2], mark[3])),
                        __builtin_bit_cast(bf16x8_t, make_uint4(seen[0], seen[1], seen[2], seen[3])), float16_t{}, 0, 0, 0);
                    const float worth = what == 1 ? __builtin_inff() : what == 2 ? -__builtin_inff() : __builtin_nanf("");
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[x][r] += hits[r] > 0.5f ? worth : 0.0f;
                }
            }
    }
    static __device__ __forceinline__ uint4 read_chunk(uint32_t lds) { return __builtin_bit_cast(uint4, *(const lds_chunk_t*)(uintptr_t)lds); }
    static __device__ __forceinline__ void write_chunk(uint32_t lds, uint4 v) { *(lds_chunk_t*)(uintptr_t)lds = __builtin_bit_cast(uint32x4_t, v); }
    static __device__ __forceinline__ bool strange(uint32_t v) { return ((v & 0x7f80u) == 0x7f80u) | ((v & 0x7f800000u) == 0x7f800000u); }
    static __device__ __forceinline__ uint32_t finite_of(uint32_t v)
    {
        return (kind(v & 0xffffu) == 0 ? v & 0xffffu : 0u) | (kind(v >> 16) == 0 ? v & 0xffff0000u : 0u);
    }
    // 0 finite, 1 infinity, 2 minus infinity, 3 NaN
    static __device__ __forceinline__ int kind(uint32_t u) { return (u & 0x7f80u) != 0x7f80u ? 0 : (u & 0x7fu) ? 3 : (u >> 15) ? 2 : 1; }
};

}  // namespace
}  // namespace moe
