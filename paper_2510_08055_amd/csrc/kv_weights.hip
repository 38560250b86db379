// The attention weight that cached tokens receive: column sums of exp(q . k / sqrt(dim) - lse), without the matrix they are sums of.
//
// Scores are computed transposed as in the attention, S = K Q^T, but here the keys stay and the rows pass by: a block holds 64 tokens' keys
// as the first operand, its four waves take 32 packed rows in turn, and a lane adds up the exponentials of its column's rows for the 16 tokens of each
// output tile that it holds.  Every token's sum belongs to one block: there are no atomics, and the order is fixed.
#include <cfloat>

#include "kv.h"

namespace moe {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float float16_t __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ uint32_t divided(uint32_t v, uint32_t d, uint32_t magic)
{
    const uint32_t q = __umulhi(v, magic);
    return q * d > v ? q - 1 : q;
}

struct Shared {
    int first[256];                // items of the chunk's sequences up to and with each
    int sums[4];
    float w[4][64];
};

template <typename T, bool FP8, int DP> struct Weights {
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int TOK = F32 && DP > 128 ? 32 : 64, NB = TOK / 32;
    static constexpr int CD = F32 ? 8 : 16, KC = DP / CD, LD = CD / 2;      // dimensions of a step of the product, steps, dimensions of a lane in it

    struct Seq {
        int row0, n, kv, held, lo;      // lo: the first token whose score changes
    };
    static __device__ __forceinline__ Seq seq_of(const WeightArgs& a, int s)
    {
        Seq q;
        q.row0 = a.c.off[s];
        const int hi = a.c.off[s + 1];
        q.n = q.row0 < 0 || hi < q.row0 || hi > a.c.T ? 0 : hi - q.row0;
        q.kv = a.c.lens[s] > 0 ? a.c.lens[s] : 0;
        const int most = a.c.max_pages << a.c.page_shift;
        q.held = q.n > 0 ? (q.kv < most ? q.kv : most) : 0;
        q.lo = 0;
        if (a.window > 0 && a.decay == 1.0f) {
            const int first = q.kv - q.n - a.window + 1;
            q.lo = first > 0 ? first & ~(TOK - 1) : 0;
        }
        return q;
    }

    static __device__ void item(const WeightArgs& a, const Seq& q, int seq, int h, int j0, Shared& sh)
    {
        const int lane = lane_id(), n = lane & 31, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
        const int D = a.c.D, shift = a.c.page_shift, G = a.G;
        auto place = [&](int j) -> int64_t {
            const int p = j >> shift;
            const int id = j < q.held ? a.c.table[(int64_t)seq * a.c.max_pages + p] : -1;
            return id < 0 || id >= a.c.n_pages ? -1 : page_row(id, a.c.Hk, h, shift, j & ((1 << shift) - 1));
        };
        bf16x8_t kb[F32 ? 1 : NB][F32 ? 1 : KC];
        float kf[F32 ? NB : 1][F32 ? KC : 1][4];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int64_t at = place(j0 + b * 32 + n), row = at < 0 ? 0 : at;       // (a token that is not there: some row, its sum is not stored)
            float sc = 1.0f;
            if constexpr (FP8) sc = scale_of(a.c.ks[row]);
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                const int d = c * CD + half * LD;
                const char* p = a.c.k + (row * D + (d < D ? d : 0)) * (FP8 ? 1 : (int)sizeof(T));
                if constexpr (F32) {
                    if constexpr (FP8) {
                        const int u = *reinterpret_cast<const int*>(p);
                        const hw_float2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8(u, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(u, true);
                        kf[b][c][0] = lo[0] * sc; kf[b][c][1] = lo[1] * sc; kf[b][c][2] = hi[0] * sc; kf[b][c][3] = hi[1] * sc;
                    } else {
                        const float4 v = *reinterpret_cast<const float4*>(p);
                        kf[b][c][0] = v.x; kf[b][c][1] = v.y; kf[b][c][2] = v.z; kf[b][c][3] = v.w;
                    }
                } else if constexpr (FP8) {      // exact: a code has 4 significant bits, its scale is a power of two
                    const uint2 u = *reinterpret_cast<const uint2*>(p);
                    const uint32_t w[2] = {u.x, u.y};
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], sc, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], sc, true);
                        kb[b][c][4 * i] = lo[0]; kb[b][c][4 * i + 1] = lo[1]; kb[b][c][4 * i + 2] = hi[0]; kb[b][c][4 * i + 3] = hi[1];
                    }
                } else {
                    kb[b][c] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4*>(p));
                }
            }
        }
        float acc[NB][16];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[b][r] = 0;

        // the rows that see some of the tokens, as packed rows; tiles of 32
        const int p0 = q.kv - q.n;
        int t_lo = a.causal && j0 > p0 ? j0 - p0 : 0, t_hi = q.n;
        if (a.window > 0) {
            const int64_t end = (int64_t)j0 + TOK - 1 - p0 + a.window;
            t_hi = end < t_hi ? (int)end : t_hi;
        }
        const int rows = q.n * G, end = t_hi * G;
        for (int r0 = (t_lo * G / 32 + wave) * 32; r0 < end; r0 += 128) {
            const int r = r0 + n;
            const bool there = r < rows;
            const int tok = !there ? 0 : G == 1 ? r : (int)divided((uint32_t)r, (uint32_t)G, a.g_magic);
            const int head = h * G + (there ? r - tok * G : 0);
            const int64_t row = q.row0 + tok;
            const float lse = a.lse[row * a.Hq + head];
            const T* src = static_cast<const T*>(a.q) + row * a.ldq + (int64_t)head * D;
            float16_t s[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) s[b] = float16_t{};
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                if (c * CD >= D) break;
                const uint4 v = *reinterpret_cast<const uint4*>(src + c * CD + half * LD);
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    if constexpr (F32) {
                        const float f[4] = {__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w)};
#pragma unroll
                        for (int x = 0; x < 4; ++x) s[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[b][c][x], f[x], s[b], 0, 0, 0);
                    } else {
                        s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kb[b][c], __builtin_bit_cast(bf16x8_t, v), s[b], 0, 0, 0);
                    }
                }
            }
            const int p = p0 + tok;
            const bool counts = there && lse != -__builtin_inff();
            const int see_hi = !counts ? 0 : a.causal ? p + 1 : 0x7fffffff, see_lo = a.window > 0 ? p - a.window + 1 : 0;
            const bool masked = __any(see_hi < j0 + TOK || see_lo > j0);
            const float lse2 = lse * kLog2e;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], a.scale2, -lse2));
                    if (masked) {
                        const int j = j0 + b * 32 + (i / 4) * 8 + 4 * half + i % 4;
                        w = j < see_hi && j >= see_lo ? w : 0.0f;
                    }
                    acc[b][i] += w;
                }
        }
        // over the columns, then the waves
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float v = acc[b][i];
#pragma unroll
                for (int d = 1; d < 32; d *= 2) v += __shfl_xor(v, d);
                if (n == 0) sh.w[wave][b * 32 + (i / 4) * 8 + 4 * half + i % 4] = v;
            }
        __syncthreads();
        if (threadIdx.x < TOK) {
            const int j = j0 + threadIdx.x;
            const int64_t at = place(j);
            if (at >= 0) {
                const int t = threadIdx.x;
                float w = (sh.w[0][t] + sh.w[1][t]) + (sh.w[2][t] + sh.w[3][t]);
                if (j < p0 && a.decay != 0.0f) w += a.decay * a.scores[at];
                a.scores[at] = w;
            }
        }
        __syncthreads();
    }
};

// Blocks take items (a sequence's tokens by TOK, and a head) in turn; 256 sequences at a time have theirs counted.
template <typename T, bool FP8, int DP> __global__ __launch_bounds__(256, 1) void weights_kernel(WeightArgs a)
{
    typedef Weights<T, FP8, DP> W;
    __shared__ Shared sh;
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    int64_t before = 0;                                  // items of earlier chunks
    for (int s0 = 0; s0 < a.c.S; s0 += 256) {
        const int s = s0 + threadIdx.x;
        int count = 0;
        if (s < a.c.S) {
            const typename W::Seq q = W::seq_of(a, s);
            count = q.held > q.lo ? (q.held - q.lo + W::TOK - 1) / W::TOK * a.c.Hk : 0;
        }
        int incl = wave_scan(count);
        if (lane == 63) sh.sums[wave] = incl;
        __syncthreads();
        for (int w = 0; w < wave; ++w) incl += sh.sums[w];
        sh.first[threadIdx.x] = incl;
        __syncthreads();
        const int total = sh.first[255];
        const int64_t behind = before % gridDim.x;
        for (int64_t i = (int64_t)blockIdx.x - behind + (blockIdx.x < behind ? gridDim.x : 0); i < total; i += gridDim.x) {
            int lo = 0, hi = 255;                        // the first sequence whose items reach past i
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (sh.first[mid] > i) hi = mid;
                else lo = mid + 1;
            }
            lo = __builtin_amdgcn_readfirstlane(lo);
            const int rem = (int)i - (lo > 0 ? sh.first[lo - 1] : 0);
            const typename W::Seq q = W::seq_of(a, s0 + lo);
            const int tile = a.c.Hk == 1 ? rem : (int)divided((uint32_t)rem, (uint32_t)a.c.Hk, a.hk_magic);
            W::item(a, q, s0 + lo, rem - tile * a.c.Hk, q.lo + tile * W::TOK, sh);
        }
        before += total;
        __syncthreads();
    }
}

template <typename T, bool FP8, int DP> hipError_t launch(WeightArgs a, hipStream_t s)
{
    // (the items of a chunk's sequences are counted in 32 bits)
    const int64_t tiles = ((int64_t)a.c.max_pages << a.c.page_shift) / Weights<T, FP8, DP>::TOK + 1;
    if (tiles * a.c.Hk > 0x7fffffff / (a.c.S < 256 ? a.c.S : 256)) return hipErrorInvalidConfiguration;
    int units = 0;
    const hipError_t e = compute_units(&units);
    if (e != hipSuccess) return e;
    a.g_magic = a.G > 1 ? (uint32_t)((((uint64_t)1 << 32) + a.G - 1) / a.G) : 0;
    a.hk_magic = a.c.Hk > 1 ? (uint32_t)((((uint64_t)1 << 32) + a.c.Hk - 1) / a.c.Hk) : 0;
    weights_kernel<T, FP8, DP><<<(unsigned)units * 2, 256, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, bool FP8> hipError_t launch_by_dim(const WeightArgs& a, hipStream_t s)
{
    if (a.c.D <= 64) return launch<T, FP8, 64>(a, s);
    if (a.c.D <= 128) return launch<T, FP8, 128>(a, s);
    return launch<T, FP8, 256>(a, s);
}

}  // namespace

hipError_t launch_kv_weights(int dtype, bool fp8, const WeightArgs& a, hipStream_t s)
{
    if (dtype == MOE_BF16) return fp8 ? launch_by_dim<bf16_t, true>(a, s) : launch_by_dim<bf16_t, false>(a, s);
    return fp8 ? launch_by_dim<float, true>(a, s) : launch_by_dim<float, false>(a, s);
}

}  // namespace moe
