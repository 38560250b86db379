#pragma once
#include "attention_plan.h"

namespace moe {
namespace {

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
//
// What bounds it: memory, where there is much to read (128 ragged histories, 719 MB, 139 us, 5.2 TB/s; 24 sequences of four drafted tokens over FP8,
// 570 MB, 120 us, 4.8 TB/s; a copy of 4 GiB moves 4.8); latency where there is little (one history of 700 tokens 9.4 us, of which the
// plan 1.5, page table and first loads 1.8, the one step of 32 tokens 2.0, the waves' join 1.1, the pieces' 1.5).
// 16 KB of keys and values are in flight to a wave; a step's products take 256 cycles of the matrix pipes at dim 128, its 16 KB 7600 of
// a SIMD's share of the memory.
// ----------------------------------------------------------------------------------------------------------------
// EXACT: the heads are DP wide, no less, and every offset within a row is a constant.
template <typename T, bool FP8, int DP, int NQ, bool EXACT> struct Few {
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
        int32_t flag;
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
        const int D = EXACT ? DP : a.c.D, shift = a.c.page_shift, Hk = a.c.Hk;
        const int begin = rg.begin, end = rg.end;
        const int per = end > begin ? (end - begin + 4 * TOK - 1) / (4 * TOK) * TOK : 0;
        const int t0 = begin + wave * per;
        const int t1 = t0 + per < end ? t0 + per : end;

        // the page table first: everything waits for it
        Entries pages;
        if (t0 < t1) pages.hold(a.c, it.seq, t0 >> shift, t1);

        // rows: what each sees, and its queries
        int see_lo[NQ], see_hi[NQ];
        Queries Q;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const Row r = row_of(a, it, rg, rg.first + i * 16 + n);
            const bool there = r.there;
            see_hi[i] = r.see_hi;
            see_lo[i] = r.see_lo;
            const T* src = static_cast<const T*>(a.q) + (int64_t)r.row * a.ldq + (int64_t)r.head * D;
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

        auto page_of = [&](int t) { return __shfl(pages.id, (t >> shift) - pages.base); };
        auto slot_of = [&](int id, int t) {
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
                const int64_t row = slot_of(page_of(tok), tok);
                const char* p = a.c.k + row * D * ESZ;
#pragma unroll
                for (int c = 0; c < KC; ++c) {
                    const int d = c * (4 * KDIM) + g * KDIM;
                    load_dwords(p + (d < D ? d : 0) * ESZ, kr[j][c]);      // (past the dimension: not used as it is)
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
                const int64_t row = slot_of(vid[j], tok);
                const char* p = a.c.v + (row * D + d) * ESZ;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    uint32_t raw[VDW];
                    load_dwords<true>(p + (int64_t)r * D * ESZ, raw);
#pragma unroll
                    for (int x = 0; x < VDW; ++x) vr[x][j * 4 + r] = raw[x];
                }
                if constexpr (FP8) vs[j] = *reinterpret_cast<const uint32_t*>(a.c.vs + row);
            }
        };

        if (t0 < t1) {
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
                // Past the dimension the queries are zero, and so are the keys: an infinity times zero would be NaN.  (fp32 loads end with the
                // dimension, a multiple of 16, and are left out, but not at 256: 32 decode rows over 2000 tokens, dim 112, us, zeros 44.5, left out
                // 43.3; dim 208 110 and 313, whose loop no longer overlaps.)
                constexpr bool LEAVE_OUT = F32 && DP <= 128;
                if (!EXACT && !LEAVE_OUT && D < DP) {
#pragma unroll
                    for (int c = 0; c < KC; ++c) {
                        if ((c + 1) * 4 * KDIM <= (DP > 64 ? DP / 2 : 16)) continue;      // (no head of this kernel is narrower)
                        if (c * (4 * KDIM) + g * KDIM < D) continue;
#pragma unroll
                        for (int x = 0; x < KDW; ++x) kr[j][c][x] = 0;
                    }
                }
                if constexpr (F32) {
#pragma unroll
                    for (int c = 0; c < KC; ++c) {
                        if (LEAVE_OUT && c * 16 >= D) break;
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
            bool gone = false;
#pragma unroll
            for (int j = 0; j < NJ; ++j) gone |= vid[j] < 0;
            const bool masked = t + TOK > rg.full_hi || t + TOK > end || t < rg.full_lo || __any(gone);
            if (more && ((t + 2 * TOK - 1) >> shift) - pages.base >= 64) pages.hold(a.c, it.seq, (t + TOK) >> shift, t1);
            // (a masked step loads the next keys at its end: what it may have to do needs the registers)
            if (more && !masked) load_k(t + TOK);

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
                clean_values(a, it, rg, t, see_lo, see_hi, vr, vs, o);
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
            if (more && masked) load_k(t + TOK);
            if (more) load_v(t + TOK);
        }

        // a wave's sums, then the block's
        const Parts parts = parts_of(a, D);
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
            const int q = threadIdx.x >> 4;
            const Row r = row_of(a, it, rg, rg.first + i * 16 + q);
            if (r.there) {
                float M = kLowest, L = 0;
#pragma unroll
                for (int w = 0; w < 4; ++w) M = fmaxf(M, sh.stats[0][w][i * 16 + q]);
#pragma unroll
                for (int w = 0; w < 4; ++w) L += sh.stats[1][w][i * 16 + q] * __builtin_amdgcn_exp2f(sh.stats[0][w][i * 16 + q] - M);
                const int part = (it.slot + it.sub * it.q.units + i) * 16 + q;
                const Finish fin = finish_row(a, r.head, M, L);
                const float to = rg.pieces > 1 ? 1.0f : fin.factor;
                for (int d = (threadIdx.x & 15) * 4; d < D; d += 64) {
                    float v[4] = {};
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float4 x = *reinterpret_cast<const float4*>(&sh.o[w][q][d]);
                        v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
                    }
                    const float4 res = make_float4(v[0] * to, v[1] * to, v[2] * to, v[3] * to);
                    if (rg.pieces > 1) store_part(parts, part, d, res);
                    else store_out<T>(a, r.row, r.head, D, d, res);
                }
                if ((threadIdx.x & 15) == 0) {
                    if (rg.pieces > 1) store_part_stats(a, part, M, L);
                    else if (a.lse) a.lse[(int64_t)r.row * a.Hq + r.head] = fin.lse;
                }
            }
        }
        if (rg.pieces > 1) join_pieces<T, DP, NQ>(a, it, rg, D, &sh.flag);
    }

    // The weights as the second product's operand.  bf16: rounded to nearest, 2^-8 of a weight at most; the sum they are divided by is that
    // of the unrounded ones, in fp32.  (A split into two bf16 halves would double the product for an output that is rounded to bf16 anyway.)
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
    // sums.  Rows that see one get it right away, as the infinity or NaN that it is; in vr they become zeros.
    static __device__ __forceinline__ bool strange(uint32_t v)
    {
        if constexpr (FP8) {        // a byte of 7f or ff: adding 1 to its low seven bits carries into the eighth
            return (((v & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
        } else if constexpr (F32) {
            return (v & 0x7f800000u) == 0x7f800000u;
        } else {
            return ((v & 0x7f80u) == 0x7f80u) | ((v & 0x7f800000u) == 0x7f800000u);
        }
    }
    static __device__ __forceinline__ uint32_t finite_of(uint32_t v)
    {
        if constexpr (FP8) {
            const uint32_t nan = ((v & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
            return v & ~(nan | (nan - (nan >> 7)));                      // (80 -> ff)
        } else if constexpr (F32) {
            return strange(v) ? 0u : v;
        } else {
            return ((v & 0x7f80u) == 0x7f80u ? 0u : v & 0xffffu) | ((v & 0x7f800000u) == 0x7f800000u ? 0u : v & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void clean_values(const AttnArgs& a, const Item& it, const Range& rg, int t, const int (&see_lo)[NQ],
                                                        const int (&see_hi)[NQ], uint32_t (&vr)[VDW][NJ * 4], uint32_t (&vs)[NJ],
                                                        float4_t (&o)[VDW][NQ][PER])
    {
        bool any = false;
#pragma unroll
        for (int s = 0; s < NJ * 4; ++s) {
#pragma unroll
            for (int x = 0; x < VDW; ++x) any |= strange(vr[x][s]);
            if constexpr (FP8) any |= ((vs[s / 4] >> (8 * (s % 4))) & 255u) == 255u;
        }
        if (!__any(any)) return;
#pragma unroll
        for (int s = 0; s < NJ * 4; ++s) {
            bool drop = false;
            if constexpr (FP8) {
                drop = ((vs[s / 4] >> (8 * (s % 4))) & 255u) == 255u;
                if (drop) vs[s / 4] = (vs[s / 4] & ~(255u << (8 * (s % 4)))) | (127u << (8 * (s % 4)));
            }
#pragma unroll
            for (int x = 0; x < VDW; ++x) vr[x][s] = drop ? 0u : finite_of(vr[x][s]);
        }
        // (rare, so slow and small: the step's tokens one by one, read again, a lane the dimensions of its outputs)
        const int g = lane_id() >> 4, D = EXACT ? DP : a.c.D;
#pragma unroll 1
        for (int tok = t; tok < t + TOK && tok < rg.hi; ++tok) {
            const int p = tok >> a.c.page_shift;
            const int id = p < a.c.max_pages ? a.c.table[(int64_t)it.seq * a.c.max_pages + p] : -1;
            if (id < 0 || id >= a.c.n_pages) continue;
            const int64_t row = page_row(id, a.c.Hk, it.head, a.c.page_shift, tok & ((1 << a.c.page_shift) - 1));
            bool nan_row = false;
            if constexpr (FP8) nan_row = a.c.vs[row] == 255;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = (g * 4 + r) * VW < D ? (g * 4 + r) * VW : 0;
                uint32_t v[VDW];
                load_dwords(a.c.v + (row * D + d) * ESZ, v);
#pragma unroll
                for (int x = 0; x < VDW; ++x)
#pragma unroll
                    for (int y = 0; y < PER; ++y) {
                        float f;
                        if constexpr (FP8) f = nan_row || ((v[x] >> (8 * y)) & 0x7fu) == 0x7fu ? __builtin_nanf("") : 0.0f;
                        else f = __uint_as_float(F32 ? v[x] : y == 0 ? v[x] << 16 : v[x] & 0xffff0000u);
                        const bool odd = (__float_as_uint(f) & 0x7f800000u) == 0x7f800000u;
#pragma unroll
                        for (int i = 0; i < NQ; ++i)
                            if (odd && tok < see_hi[i] && tok >= see_lo[i]) o[x][i][y][r] += f;
                    }
            }
        }
    }
};

}  // namespace
}  // namespace moe
