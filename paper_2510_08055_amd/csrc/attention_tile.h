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
// ----------------------------------------------------------------------------------------------------------------
constexpr int kManyRows = 128;

template <bool FP8, int DP> struct Many {
    static constexpr int TOK = 64;
    static constexpr int ROWB = DP * 2;              // bytes of a token's row in LDS
    static constexpr int CH = DP / 8;                // its 16-byte chunks
    static constexpr int HALF = TOK * ROWB;          // keys, then values
    static constexpr int STAGE = 2 * HALF;
    static constexpr size_t LDS = 2 * STAGE;
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

    // The step's source in the cache: an address per group of 8 tokens (pages hold whole groups), and which groups are there.
    struct Step {
        int t;
        uint32_t there;              // bit i: tokens t + 8 i .. t + 8 i + 7
    };

    typedef short short4_t __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) short4_t lds_short4_t;
    static __device__ __forceinline__ uint2 read_transposed(uint32_t lds)
    {
        return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t*)(uintptr_t)lds));
    }

    static __device__ __forceinline__ void run(const AttnArgs& a, const Item& it, char* smem)
    {
        const Range rg = range_of(a, it);
        if (it.sub >= rg.pieces) return;
        const int lane = lane_id(), n = lane & 31, h = lane >> 5;
        const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
        const int D = a.c.D, shift = a.c.page_shift, Hk = a.c.Hk;
        const uint32_t lds0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds_address(smem));

        const Row me = row_of(a, it, rg, rg.first + wave * 32 + n);
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

        // ---- staging ----
        Entries pages;
        const int64_t head_row = (int64_t)it.head << shift;
        auto step_at = [&](int t) {
            if (((t + TOK - 1) >> shift) - pages.base >= 64) pages.hold(a.c, it.seq, t >> shift, rg.end);
            const unsigned long long ok = __ballot(pages.id >= 0);
            Step s;
            s.t = t;
            s.there = 0;
#pragma unroll
            for (int i = 0; i < TOK / 8; ++i) s.there |= (uint32_t)((ok >> (((t + 8 * i) >> shift) - pages.base)) & 1) << i;
            return s;
        };
        // byte offset of token t's row (of a group of tokens that the wave shares) in the pages; row_bytes: of a cached row
        auto group_row = [&](int t) {
            int id = __builtin_amdgcn_readlane(pages.id, (t >> shift) - pages.base);
            id = id < 0 ? 0 : id;
            return ((((int64_t)id * Hk) << shift) + head_row + (t & ((1 << shift) - 1)));
        };
        // bf16: straight into LDS, 64 / CH tokens to a wave's load
        constexpr int TPL = 64 / CH;
        auto stage = [&](const Step& s, uint32_t base) {
            const int tl = lane / CH, c = lane % CH;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int t = (wave * LOADS + i) * TPL;              // of the step; the same 8-token group for all of the load
                const int64_t row = group_row(s.t + t);
                // (chunks past the dimension: keys meet zeros there, values go to outputs that are not stored)
                const int chunk = c ^ swz(t + tl);
                const uint32_t off = (uint32_t)(tl * D * 2 + (chunk * 8 < D ? chunk * 16 : 0));
                const char* k = uniform(a.c.k + row * D * 2);
                const char* v = uniform(a.c.v + row * D * 2);
                load_lds_16_base(k, off, base + t * ROWB);
                load_lds_16_base(v, off, base + HALF + t * ROWB);
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
#pragma unroll
            for (int i = 0; i < FL; ++i) {
                const int t = (wave * FL + i) * TPW + tl;
                int id = __shfl(pages.id, ((s.t + t) >> shift) - pages.base);
                const int64_t row = page_row(id < 0 ? 0 : id, Hk, it.head, shift, (s.t + t) & ((1 << shift) - 1));
                const int64_t off = row * D + (c * 16 < D ? c * 16 : 0);
                raw[i][0] = *reinterpret_cast<const uint4*>(a.c.k + off);
                raw[i][1] = *reinterpret_cast<const uint4*>(a.c.v + off);
                raw_scale[i][0] = a.c.ks[row];
                raw_scale[i][1] = a.c.vs[row];
            }
        };
        auto widen = [&](char* base) {
            const int tl = lane / LPT, c = lane % LPT;
#pragma unroll
            for (int i = 0; i < FL; ++i) {
                const int t = (wave * FL + i) * TPW + tl;
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

        // ---- operand addresses (relative to a stage) ----
        // keys: token 32 b + n, chunk 2 s + h
        const int k_row = n * ROWB, k_swz = swz(n);
        // values: tokens 16 s + 8 u + 4 h + (lane % 16) / 4, dimensions 32 nb + 16 (lane / 16 % 2) + 4 (lane % 4): see read_transposed
        const int v_tok = 4 * h + ((lane & 15) >> 2), v_chunk = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
        const int v_row = v_tok * ROWB + (lane & 1) * 8;
        auto v_at = [&](int s, int u, int nb) {
            const int t = 8 * u + v_tok;                             // (16 s does not change the swizzle)
            return (uint32_t)(v_row + (16 * s + 8 * u) * ROWB + ((v_chunk + 4 * nb) ^ swz(t)) * 16);
        };

        float m = kLowest, l = 0;
        float16_t o[NB];
#pragma unroll
        for (int x = 0; x < NB; ++x) o[x] = float16_t{};

        Step cur{rg.begin, 0};
        if (rg.begin < rg.end) {
            pages.hold(a.c, it.seq, rg.begin >> shift, rg.end);
            cur = step_at(rg.begin);
            if constexpr (FP8) {
                fetch(cur);
                widen(smem);
            } else {
                stage(cur, lds0);
            }
        }
        const bool idle = rg.first + wave * 32 >= rg.rows;           // a wave whose rows are none stages all the same
        uint32_t at = 0;                                             // byte offset of the step's stage
        while (cur.t < rg.end) {
            if constexpr (FP8) wait_lds_reads();
            else wait_vmcnt<0>();
            block_barrier();
            Step next{cur.t + TOK, 0};
            const bool more = next.t < rg.end;
            if (more) {
                next = step_at(next.t);
                if constexpr (FP8) fetch(next);
                else stage(next, lds0 + (at ^ STAGE));
            }
            if (!idle) {
                const char* kb = smem + at;
                float16_t s[2];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    s[b] = float16_t{};
#pragma unroll
                    for (int c = 0; c < DP / 16; ++c) {
                        const uint4 kf = *reinterpret_cast<const uint4*>(kb + b * 32 * ROWB + k_row + (((2 * c + h) ^ k_swz) * 16));
                        s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf), qf[c], s[b], 0, 0, 0);
                    }
                }
                const bool masked = cur.t + TOK > rg.full_hi || cur.t < rg.full_lo || cur.there != 0xffu;
                float top = -__builtin_inff();
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        float x = s[b][r] * a.scale2;
                        if (masked) {
                            const int grp = b * 4 + r / 4, tok = cur.t + grp * 8 + 4 * h + r % 4;
                            if (!(((cur.there >> grp) & 1) && tok < me.see_hi && tok >= me.see_lo)) x = -__builtin_inff();
                        }
                        s[b][r] = x;
                        top = fmaxf(top, x);
                    }
                top = swap_max(top);
                // (the reference of the exponentials follows the maximum only when that has grown by more than 8, see attention_few.h)
                if (__any(top > m + 8.0f)) {
                    const float to = fmaxf(top, m), f = __builtin_amdgcn_exp2f(m - to);
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
                        const float p0 = __builtin_amdgcn_exp2f(s[k / 2][(k % 2) * 8 + 2 * i] - m);
                        const float p1 = __builtin_amdgcn_exp2f(s[k / 2][(k % 2) * 8 + 2 * i + 1] - m);
                        l += p0;
                        l += p1;
                        u[i] = pack_bf16x2(p0, p1);
                    }
                    w[k] = __builtin_bit_cast(bf16x8_t, make_uint4(u[0], u[1], u[2], u[3]));
                }
                const uint32_t vb = lds0 + at + HALF;
                if (!masked) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int x = 0; x < NB; ++x) {
                            const uint2 lo = read_transposed(vb + v_at(k, 0, x)), hi = read_transposed(vb + v_at(k, 1, x));
                            o[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                                __builtin_bit_cast(bf16x8_t, make_uint4(lo.x, lo.y, hi.x, hi.y)), w[k], o[x], 0, 0, 0);
                        }
                } else {
                    careful_values(cur, rg, me, vb, v_at, w, o);
                }
            }
            if constexpr (FP8)
                if (more) widen(smem + (at ^ STAGE));
            at ^= STAGE;
            cur = next;
        }

        // results
        l = swap_sum(l);
        const Finish fin = finish_row(a, me.head, m, l);
        const float f = rg.pieces > 1 ? 1.0f : fin.factor;
        const int64_t part = (int64_t)(it.slot + it.sub * it.q.units) * 16 + wave * 32 + n;
        if (me.there) {
#pragma unroll
            for (int x = 0; x < NB; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int d = x * 32 + r * 8 + h * 4;
                    const float4 v = make_float4(o[x][4 * r] * f, o[x][4 * r + 1] * f, o[x][4 * r + 2] * f, o[x][4 * r + 3] * f);
                    if (d < D) {
                        if (rg.pieces > 1) store_part(a, part, d, v);
                        else store_out<bf16_t>(a, me.row, me.head, d, v);
                    }
                }
            if (h == 0) {
                if (rg.pieces > 1) store_part_stats(a, part, m, l);
                else if (a.lse) a.lse[(int64_t)me.row * a.Hq + me.head] = fin.lse;
            }
        }
        if (rg.pieces > 1) {
            __syncthreads();                                         // the flag shares the stages' memory
            join_pieces<bf16_t, DP>(a, it, rg, reinterpret_cast<int32_t*>(smem));
        }
    }

    // The second product for a step whose tokens not every row sees: values of tokens that are not there, or that no row sees, are
    // zeros whatever the cache holds, and those that are not finite (a weight of zero would not keep them out) go to the rows
    // that see them as the infinity or NaN that they are.
    template <typename At>
    static __device__ __forceinline__ void careful_values(const Step& cur, const Range& rg, const Row& me, uint32_t vb, At v_at,
                                                          const bf16x8_t (&w)[4], float16_t (&o)[NB])
    {
        const int h = lane_id() >> 5;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t keep[4], seen[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                keep[i] = seen[i] = 0;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int grp = 2 * k + i / 2, tok = cur.t + grp * 8 + 4 * h + (i % 2) * 2 + e;
                    const bool there = (cur.there >> grp) & 1;
                    if (there && tok < rg.hi) keep[i] |= 0xffffu << (16 * e);
                    if (there && tok < me.see_hi && tok >= me.see_lo) seen[i] |= 0x3f80u << (16 * e);
                }
            }
#pragma unroll
            for (int x = 0; x < NB; ++x) {
                const uint2 lo = read_transposed(vb + v_at(k, 0, x)), hi = read_transposed(vb + v_at(k, 1, x));
                uint32_t v[4] = {lo.x & keep[0], lo.y & keep[1], hi.x & keep[2], hi.y & keep[3]};
                bool strange = false;
#pragma unroll
                for (int i = 0; i < 4; ++i) strange |= (v[i] & 0x7f80u) == 0x7f80u || (v[i] & 0x7f800000u) == 0x7f800000u;
                if (__any(strange)) {
#pragma unroll 1
                    for (int what = 1; what <= 3; ++what) {          // infinity, minus infinity, NaN
                        uint32_t mark[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            mark[i] = 0;
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (kind((v[i] >> (16 * e)) & 0xffffu) == what) mark[i] |= 0x3f80u << (16 * e);
                        }
                        const float16_t hits = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            __builtin_bit_cast(bf16x8_t, make_uint4(mark[0], mark[1], mark[2], mark[3])),
                            __builtin_bit_cast(bf16x8_t, make_uint4(seen[0], seen[1], seen[2], seen[3])), float16_t{}, 0, 0, 0);
                        const float worth = what == 1 ? __builtin_inff() : what == 2 ? -__builtin_inff() : __builtin_nanf("");
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[x][r] += hits[r] > 0.5f ? worth : 0.0f;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (kind(v[i] & 0xffffu) != 0) v[i] &= 0xffff0000u;
                        if (kind(v[i] >> 16) != 0) v[i] &= 0xffffu;
                    }
                }
                o[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, make_uint4(v[0], v[1], v[2], v[3])), w[k], o[x],
                                                               0, 0, 0);
            }
        }
    }
    // 0 finite, 1 infinity, 2 minus infinity, 3 NaN
    static __device__ __forceinline__ int kind(uint32_t u) { return (u & 0x7f80u) != 0x7f80u ? 0 : (u & 0x7fu) ? 3 : (u >> 15) ? 2 : 1; }
};

}  // namespace
}  // namespace moe
