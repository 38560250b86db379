// Writing rows into the pages of a key/value cache and reading them back.  Both move bytes: a row and head is read once and
// written once, in 16-byte pieces, by a group of lanes that covers it; what bounds them is the launch and one chain of
// dependent loads (row -> sequence -> page -> slot) in small batches, memory in large ones.
#include "kv.h"

namespace moe {
namespace {

// The sequence of row `row` (the same in every lane): how many of off[1 .. S] are <= row.  64 entries at a time, so up to 64
// sequences take one step, up to 4096 two; a binary search would take a dependent load for every doubling.
__device__ __forceinline__ int find_sequence(const int32_t* __restrict__ off, int S, int row)
{
    const int lane = lane_id();
    int lo = 0, hi = S;
    while (hi - lo > 64) {
        const int step = (hi - lo + 63) / 64;
        const int i = lo + (lane + 1) * step - 1;
        const bool below = i < hi && off[1 + (i < hi ? i : hi - 1)] <= row;
        const int n = __popcll(__ballot(below));
        lo += n * step;
        if (lo > hi) lo = hi;
        if (lo + step - 1 < hi) hi = lo + step - 1;
    }
    const int i = lo + lane;
    const bool below = i < hi && off[1 + (i < hi ? i : (hi > 0 ? hi - 1 : 0))] <= row;
    return lo + __popcll(__ballot(below));
}

// Where the row of lane's vector lies: its row index among the pages' rows, or -1 where the token is not there.
// first: the wave's first row; rows of a wave differ by little, so a lane steps on from that row's sequence.
__device__ __forceinline__ int64_t find_slot(const KVView& c, int first, int row, int h)
{
    int s = find_sequence(c.off, c.S, first);
    while (s < c.S && c.off[s + 1] <= row) ++s;
    if (s >= c.S) return -1;
    const int len = c.lens[s];
    const int pos = (len > 0 ? len : 0) - (c.off[s + 1] - row);
    const int p = pos >> c.page_shift;
    if (pos < 0 || p >= c.max_pages) return -1;
    const int id = c.table[(int64_t)s * c.max_pages + p];
    if (id < 0 || id >= c.n_pages) return -1;
    return page_row(id, c.Hk, h, c.page_shift, pos & ((1 << c.page_shift) - 1));
}

struct Vec {
    int row, h;      // row of the batch, key/value head
    bool value;      // a row of v
    int first;       // row of the wave's first vector
    int piece;       // the lane's place among the vector's lanes
    bool valid;
};
// The vectors (row, k or v, head) of a batch in that order, LPR lanes to each.
template <int LPR> __device__ __forceinline__ Vec my_vector(const KVView& c)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t vec = at / LPR;
    const int64_t vec0 = (at - lane_id()) / LPR;
    const int per_row = 2 * c.Hk;
    Vec v;
    v.piece = (int)(at % LPR);
    v.row = (int)(vec / per_row);
    const int r = (int)(vec - (int64_t)v.row * per_row);
    v.value = r >= c.Hk;
    v.h = v.value ? r - c.Hk : r;
    v.first = __builtin_amdgcn_readfirstlane((int)(vec0 / per_row));
    v.valid = v.row < c.T;
    return v;
}

template <typename T> __device__ __forceinline__ void load8(const T* p, float (&x)[8])
{
    if constexpr (sizeof(T) == 2) {
        const uint4 raw = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
}

// As it is: 16 bytes to a lane.  esz: bytes of an element.
template <int LPR> __global__ __launch_bounds__(256) void append_kernel(KVView c, const char* __restrict__ k, int64_t ldk,
                                                                        const char* __restrict__ v, int64_t ldv, int esz)
{
    const Vec t = my_vector<LPR>(c);
    const int bytes = c.D * esz;
    const bool mine = t.valid && t.piece * 16 < bytes;
    uint4 x = {};
    if (mine) {
        const char* src = t.value ? v + (int64_t)t.row * ldv * esz : k + (int64_t)t.row * ldk * esz;
        x = *reinterpret_cast<const uint4*>(src + (int64_t)t.h * bytes + t.piece * 16);
    }
    const int64_t at = find_slot(c, t.first, t.row, t.h);
    if (mine && at >= 0) *reinterpret_cast<uint4*>((t.value ? c.v : c.k) + at * bytes + t.piece * 16) = x;
}

// As FP8 codes: 8 elements to a lane.
template <typename T, int LPR> __global__ __launch_bounds__(256) void append_fp8_kernel(KVView c, const T* __restrict__ k, int64_t ldk,
                                                                                        const T* __restrict__ v, int64_t ldv)
{
    const Vec t = my_vector<LPR>(c);
    const bool mine = t.valid && t.piece * 8 < c.D;
    float x[8] = {};
    if (mine) load8((t.value ? v + (int64_t)t.row * ldv : k + (int64_t)t.row * ldk) + t.h * c.D + t.piece * 8, x);
    const int64_t at = find_slot(c, t.first, t.row, t.h);
    // |x| as integers: they order like the values, and everything that is not finite comes last
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
        top = a > top ? a : top;
    }
#pragma unroll
    for (int d = 1; d < LPR; d *= 2) {
        const uint32_t o = (uint32_t)__shfl_xor((int)top, d);
        top = o > top ? o : top;
    }
    // amax = m 2^(E - 126) with m in [1/2, 1): e = E - 126 - 9 if m <= 448 / 512, one more otherwise
    const bool bad = top >= 0x7f800000u;
    int e = (int)(top >> 23) - 135 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = e < -100 ? -100 : e;
    if (top == 0) e = -9;
    if (!mine || at < 0) return;
    uint32_t lo = 0, hi = 0;
    if (bad) {
        lo = hi = 0x7f7f7f7fu;
    } else {
        // (a power of two is exact, except where it takes a value below the smallest normal one, far below the smallest code)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_ldexpf(x[i], -e);
        lo = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
        lo = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], (int)lo, true);
        hi = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], 0, false);
        hi = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], (int)hi, true);
    }
    *reinterpret_cast<uint2*>((t.value ? c.v : c.k) + at * c.D + t.piece * 8) = make_uint2(lo, hi);
    if (t.piece == 0) (t.value ? c.vs : c.ks)[at] = (uint8_t)(bad ? 255 : e + 127);
}

template <int LPR> __global__ __launch_bounds__(256) void gather_kernel(KVView c, char* __restrict__ k, int64_t ldk, char* __restrict__ v,
                                                                        int64_t ldv, int esz)
{
    const Vec t = my_vector<LPR>(c);
    const int bytes = c.D * esz;
    const int64_t at = find_slot(c, t.first, t.row, t.h);
    if (!t.valid || t.piece * 16 >= bytes) return;
    uint4 x = {};
    if (at >= 0) x = *reinterpret_cast<const uint4*>((t.value ? c.v : c.k) + at * bytes + t.piece * 16);
    char* dst = t.value ? v + (int64_t)t.row * ldv * esz : k + (int64_t)t.row * ldk * esz;
    *reinterpret_cast<uint4*>(dst + (int64_t)t.h * bytes + t.piece * 16) = x;
}

template <typename T, int LPR> __global__ __launch_bounds__(256) void gather_fp8_kernel(KVView c, T* __restrict__ k, int64_t ldk,
                                                                                        T* __restrict__ v, int64_t ldv)
{
    const Vec t = my_vector<LPR>(c);
    const int64_t at = find_slot(c, t.first, t.row, t.h);
    if (!t.valid || t.piece * 8 >= c.D) return;
    float x[8] = {};
    if (at >= 0) {
        const uint2 w = *reinterpret_cast<const uint2*>((t.value ? c.v : c.k) + at * c.D + t.piece * 8);
        const float s = scale_of((t.value ? c.vs : c.ks)[at]);
        const hw_float2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.x, true);
        const hw_float2_t d = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, false), e = __builtin_amdgcn_cvt_pk_f32_fp8((int)w.y, true);
        x[0] = a[0] * s; x[1] = a[1] * s; x[2] = b[0] * s; x[3] = b[1] * s;
        x[4] = d[0] * s; x[5] = d[1] * s; x[6] = e[0] * s; x[7] = e[1] * s;
    }
    T* dst = (t.value ? v + (int64_t)t.row * ldv : k + (int64_t)t.row * ldk) + t.h * c.D + t.piece * 8;
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                                                    pack_bf16x2(x[6], x[7]));
    } else {
        reinterpret_cast<float4*>(dst)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4*>(dst)[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
}

// Lanes to a vector of n pieces: the next power of two, 8 at least.
template <typename F> hipError_t by_lanes(int n, F f)
{
    if (n <= 8) return f(std::integral_constant<int, 8>());
    if (n <= 16) return f(std::integral_constant<int, 16>());
    if (n <= 32) return f(std::integral_constant<int, 32>());
    return f(std::integral_constant<int, 64>());
}
inline unsigned blocks_for(const KVView& c, int lanes)
{
    return (unsigned)(((int64_t)c.T * 2 * c.Hk * lanes + 255) / 256);
}

}  // namespace

hipError_t launch_kv_append(int dtype, bool fp8, const KVView& c, const void* k, int64_t ldk, const void* v, int64_t ldv, hipStream_t s)
{
    const int esz = dtype == MOE_BF16 ? 2 : 4;
    if (!fp8)
        return by_lanes(c.D * esz / 16, [&](auto lpr) {
            constexpr int L = decltype(lpr)::value;
            append_kernel<L><<<blocks_for(c, L), 256, 0, s>>>(c, static_cast<const char*>(k), ldk, static_cast<const char*>(v), ldv, esz);
            return hipGetLastError();
        });
    return by_lanes(c.D / 8, [&](auto lpr) {
        constexpr int L = decltype(lpr)::value;
        if (dtype == MOE_BF16)
            append_fp8_kernel<bf16_t, L><<<blocks_for(c, L), 256, 0, s>>>(c, static_cast<const bf16_t*>(k), ldk, static_cast<const bf16_t*>(v), ldv);
        else
            append_fp8_kernel<float, L><<<blocks_for(c, L), 256, 0, s>>>(c, static_cast<const float*>(k), ldk, static_cast<const float*>(v), ldv);
        return hipGetLastError();
    });
}

hipError_t launch_kv_gather(int dtype, bool fp8, const KVView& c, void* k, int64_t ldk, void* v, int64_t ldv, hipStream_t s)
{
    const int esz = dtype == MOE_BF16 ? 2 : 4;
    if (!fp8)
        return by_lanes(c.D * esz / 16, [&](auto lpr) {
            constexpr int L = decltype(lpr)::value;
            gather_kernel<L><<<blocks_for(c, L), 256, 0, s>>>(c, static_cast<char*>(k), ldk, static_cast<char*>(v), ldv, esz);
            return hipGetLastError();
        });
    return by_lanes(c.D / 8, [&](auto lpr) {
        constexpr int L = decltype(lpr)::value;
        if (dtype == MOE_BF16)
            gather_fp8_kernel<bf16_t, L><<<blocks_for(c, L), 256, 0, s>>>(c, static_cast<bf16_t*>(k), ldk, static_cast<bf16_t*>(v), ldv);
        else
            gather_fp8_kernel<float, L><<<blocks_for(c, L), 256, 0, s>>>(c, static_cast<float*>(k), ldk, static_cast<float*>(v), ldv);
        return hipGetLastError();
    });
}

}  // namespace moe
