// Writing rows into the pages of a key/value cache and reading them back.  Both move bytes: a row and head is read once and
// written once, in 16-byte pieces, by a group of lanes that covers it; what bounds them is the launch and one chain of
// dependent loads (ends of sequences -> page -> slot) in small batches, memory in large ones.  Kernel times: 32 rows of a decode step 3.0 us; 8320
// rows quantised (26 MB) 7.7; three bf16 histories read back (24 MB) 4.8, 16 FP8 ones (170 MB) 27 with what the last-level cache
// holds of them, 36 cold (4.7 TB/s).  Four vectors of a row to a wave: two 46 us, eight 41 on the last.
#include "kv.h"

namespace moe {
namespace {

// A wave's share of a batch: 64 / LPR consecutive rows, LPR lanes to each, and R of a row's 2 Hk vectors (keys of all heads, then
// values).  Consecutive tokens of a head lie side by side in a page, so a wave reads (or writes) whole stretches of it and whole
// vectors of the rows, and a row's place is looked up once for its R vectors, all of which are in flight together.
constexpr int R = 4;
struct Share {
    int row, first;      // this lane's row, the wave's first
    int piece;           // the lane's place among its vector's lanes
    int r0;              // the first vector
    bool valid;
};
template <int LPR> __device__ __forceinline__ Share my_share(const KVView& c)
{
    const int parts = (2 * c.Hk + R - 1) / R;
    const int wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
    const int group = wave / parts;
    Share s;
    s.first = group * (64 / LPR);
    s.row = s.first + lane_id() / LPR;
    s.piece = lane_id() % LPR;
    s.r0 = (wave - group * parts) * R;
    s.valid = s.row < c.T;
    return s;
}

// Where the row's token lies: the index of its row for head 0 among the pages' rows, or -1 where it is not there.
// The row's sequence is found 64 ends of sequences at a time, so up to 64 sequences take one load, up to 4096 two (a binary search
// would take a dependent one for every doubling); the last 64 stay in the lanes, with the lengths, for all rows of the wave.
template <int LPR> __device__ __forceinline__ int64_t find_slot(const KVView& c, const Share& t)
{
    const int lane = lane_id();
    int lo = 0, hi = c.S;       // how many of off[1 .. S] are <= first
    while (hi - lo > 64) {
        const int step = (hi - lo + 63) / 64;
        const int i = lo + (lane + 1) * step - 1;
        const bool below = i < hi && c.off[1 + (i < hi ? i : hi - 1)] <= t.first;
        lo += __popcll(__ballot(below)) * step;
        if (lo > hi) lo = hi;
        if (lo + step - 1 < hi) hi = lo + step - 1;
    }
    const int mine = lo + lane < c.S ? lo + lane : c.S - 1;
    const int end = lo + lane < c.S ? c.off[1 + mine] : 0x7fffffff, held = c.lens[mine];
    int s = 0;
#pragma unroll
    for (int k = 0; k < 64 / LPR; ++k) {
        const int n = __popcll(__ballot(end <= t.first + k));
        s = lane / LPR == k ? n : s;
    }
    int until = __shfl(end, s & 63), len = __shfl(held, s & 63);
    s += lo;
    // 64 sequences and more between two rows of the wave, empty ones: the lane looks by halves (rows in the first and the last of 256 / 4096 / 65536
    // slots 3.6 / 4.0 / 4.8 us, in neighbouring ones 3; one by one 22 / 414 / -).
    if (s >= lo + 64) {
        for (int end = c.S; s < end;) {
            const int mid = s + (end - s) / 2;
            if (c.off[mid + 1] <= t.row) s = mid + 1;
            else end = mid;
        }
        until = s < c.S ? c.off[s + 1] : 0;
        len = s < c.S ? c.lens[s] : 0;
    }
    if (s >= c.S) return -1;
    const int pos = (len > 0 ? len : 0) - (until - t.row);
    const int p = pos >> c.page_shift;
    if (pos < 0 || p >= c.max_pages) return -1;
    const int id = c.table[(int64_t)s * c.max_pages + p];
    if (id < 0 || id >= c.n_pages) return -1;
    return page_row(id, c.Hk, 0, c.page_shift, pos & ((1 << c.page_shift) - 1));
}

// Vector r of a row: of the values?, and its head.
__device__ __forceinline__ bool is_value(const KVView& c, int r) { return r >= c.Hk; }
__device__ __forceinline__ int head_of(const KVView& c, int r) { return r >= c.Hk ? r - c.Hk : r; }

// 16 bytes that go out as a stream: rows read back are as large as what they are read from, and whoever wants them comes later
// (16 FP8 histories, 165 MB, with cold caches 39.8 -> 37.4 us).
__device__ __forceinline__ void store_stream(void* p, uint4 v)
{
    typedef uint32_t uint32x4_t __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(__builtin_bit_cast(uint32x4_t, v), static_cast<uint32x4_t*>(p));
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
    const Share t = my_share<LPR>(c);
    const int bytes = c.D * esz;
    const bool mine = t.valid && t.piece * 16 < bytes;
    uint4 x[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int r = t.r0 + i;
        x[i] = make_uint4(0, 0, 0, 0);
        if (mine && r < 2 * c.Hk) {
            const char* src = is_value(c, r) ? v + (int64_t)t.row * ldv * esz : k + (int64_t)t.row * ldk * esz;
            x[i] = *reinterpret_cast<const uint4*>(src + (int64_t)head_of(c, r) * bytes + t.piece * 16);
        }
    }
    const int64_t at = find_slot<LPR>(c, t);
    if (!mine || at < 0) return;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int r = t.r0 + i;
        if (r < 2 * c.Hk)
            *reinterpret_cast<uint4*>((is_value(c, r) ? c.v : c.k) + (at + ((int64_t)head_of(c, r) << c.page_shift)) * bytes + t.piece * 16) = x[i];
    }
}

// As FP8 codes: 8 elements to a lane.
template <typename T, int LPR> __global__ __launch_bounds__(256) void append_fp8_kernel(KVView c, const T* __restrict__ k, int64_t ldk,
                                                                                        const T* __restrict__ v, int64_t ldv)
{
    const Share t = my_share<LPR>(c);
    const bool mine = t.valid && t.piece * 8 < c.D;
    float x[R][8] = {};
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int r = t.r0 + i;
        if (mine && r < 2 * c.Hk)
            load8((is_value(c, r) ? v + (int64_t)t.row * ldv : k + (int64_t)t.row * ldk) + head_of(c, r) * c.D + t.piece * 8, x[i]);
    }
    const int64_t at = find_slot<LPR>(c, t);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int r = t.r0 + i;
        // |x| as integers: they order like the values, and everything that is not finite comes last
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t a = __float_as_uint(x[i][e]) & 0x7fffffffu;
            top = a > top ? a : top;
        }
#pragma unroll
        for (int d = 1; d < LPR; d *= 2) {
            const uint32_t o = (uint32_t)__shfl_xor((int)top, d);
            top = o > top ? o : top;
        }
        if (!mine || at < 0 || r >= 2 * c.Hk) continue;
        // amax = m 2^(E - 126) with m in [1/2, 1): e = E - 126 - 9 if m <= 448 / 512, one more otherwise
        const bool bad = top >= 0x7f800000u;
        int e = (int)(top >> 23) - 135 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
        e = e < -100 ? -100 : e;
        if (top == 0) e = -9;
        uint32_t lo = 0x7f7f7f7fu, hi = 0x7f7f7f7fu;
        if (!bad) {
            // (a power of two is exact, except where it takes a value below the smallest normal one, far below the smallest code)
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = __builtin_amdgcn_ldexpf(x[i][j], -e);
            lo = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
            lo = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], (int)lo, true);
            hi = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
            hi = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], (int)hi, true);
        }
        const int64_t to = at + ((int64_t)head_of(c, r) << c.page_shift);
        *reinterpret_cast<uint2*>((is_value(c, r) ? c.v : c.k) + to * c.D + t.piece * 8) = make_uint2(lo, hi);
        if (t.piece == 0) (is_value(c, r) ? c.vs : c.ks)[to] = (uint8_t)(bad ? 255 : e + 127);
    }
}

template <int LPR> __global__ __launch_bounds__(256) void gather_kernel(KVView c, char* __restrict__ k, int64_t ldk, char* __restrict__ v,
                                                                        int64_t ldv, int esz)
{
    const Share t = my_share<LPR>(c);
    const int bytes = c.D * esz;
    const int64_t at = find_slot<LPR>(c, t);
    if (!t.valid || t.piece * 16 >= bytes) return;
    uint4 x[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int r = t.r0 + i;
        x[i] = make_uint4(0, 0, 0, 0);
        if (at >= 0 && r < 2 * c.Hk)
            x[i] = *reinterpret_cast<const uint4*>((is_value(c, r) ? c.v : c.k) + (at + ((int64_t)head_of(c, r) << c.page_shift)) * bytes + t.piece * 16);
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int r = t.r0 + i;
        if (r >= 2 * c.Hk) break;
        char* dst = is_value(c, r) ? v + (int64_t)t.row * ldv * esz : k + (int64_t)t.row * ldk * esz;
        store_stream(dst + (int64_t)head_of(c, r) * bytes + t.piece * 16, x[i]);
    }
}

template <typename T, int LPR> __global__ __launch_bounds__(256) void gather_fp8_kernel(KVView c, T* __restrict__ k, int64_t ldk,
                                                                                        T* __restrict__ v, int64_t ldv)
{
    const Share t = my_share<LPR>(c);
    const int64_t at = find_slot<LPR>(c, t);
    if (!t.valid || t.piece * 8 >= c.D) return;
    uint2 w[R];
    uint32_t sb[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int r = t.r0 + i;
        w[i] = make_uint2(0, 0);
        sb[i] = 127;
        if (at >= 0 && r < 2 * c.Hk) {
            const int64_t from = at + ((int64_t)head_of(c, r) << c.page_shift);
            w[i] = *reinterpret_cast<const uint2*>((is_value(c, r) ? c.v : c.k) + from * c.D + t.piece * 8);
            sb[i] = (is_value(c, r) ? c.vs : c.ks)[from];
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int r = t.r0 + i;
        if (r >= 2 * c.Hk) break;
        const float s = scale_of(sb[i]);
        float x[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int u = (int)(h == 0 ? w[i].x : w[i].y);
            const hw_float2_t a = __builtin_amdgcn_cvt_pk_f32_fp8(u, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(u, true);
            x[4 * h] = a[0] * s; x[4 * h + 1] = a[1] * s; x[4 * h + 2] = b[0] * s; x[4 * h + 3] = b[1] * s;
        }
        T* dst = (is_value(c, r) ? v + (int64_t)t.row * ldv : k + (int64_t)t.row * ldk) + head_of(c, r) * c.D + t.piece * 8;
        if constexpr (sizeof(T) == 2) {
            store_stream(dst, make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])));
        } else {
            store_stream(dst, __builtin_bit_cast(uint4, make_float4(x[0], x[1], x[2], x[3])));
            store_stream(dst + 4, __builtin_bit_cast(uint4, make_float4(x[4], x[5], x[6], x[7])));
        }
    }
}

// f with the lanes to a vector of n pieces (the next power of two, 8 at least) and the blocks that they take for the batch.
template <typename F> hipError_t by_lanes(const KVView& c, int n, F f)
{
    auto with = [&](auto lanes) {
        const int64_t groups = ((int64_t)c.T * decltype(lanes)::value + 63) / 64, parts = (2 * c.Hk + R - 1) / R;
        const int64_t blocks = (groups * parts + 3) / 4;
        return blocks <= kMaxBlocks ? f(lanes, (unsigned)blocks) : hipErrorInvalidConfiguration;
    };
    if (n <= 8) return with(std::integral_constant<int, 8>());
    if (n <= 16) return with(std::integral_constant<int, 16>());
    if (n <= 32) return with(std::integral_constant<int, 32>());
    return with(std::integral_constant<int, 64>());
}

}  // namespace

hipError_t launch_kv_append(int dtype, bool fp8, const KVView& c, const void* k, int64_t ldk, const void* v, int64_t ldv, hipStream_t s)
{
    const int esz = dtype == MOE_BF16 ? 2 : 4;
    if (!fp8)
        return by_lanes(c, c.D * esz / 16, [&](auto lpr, unsigned blocks) {
            constexpr int L = decltype(lpr)::value;
            append_kernel<L><<<blocks, 256, 0, s>>>(c, static_cast<const char*>(k), ldk, static_cast<const char*>(v), ldv, esz);
            return hipGetLastError();
        });
    return by_lanes(c, c.D / 8, [&](auto lpr, unsigned blocks) {
        constexpr int L = decltype(lpr)::value;
        if (dtype == MOE_BF16)
            append_fp8_kernel<bf16_t, L><<<blocks, 256, 0, s>>>(c, static_cast<const bf16_t*>(k), ldk, static_cast<const bf16_t*>(v), ldv);
        else
            append_fp8_kernel<float, L><<<blocks, 256, 0, s>>>(c, static_cast<const float*>(k), ldk, static_cast<const float*>(v), ldv);
        return hipGetLastError();
    });
}

hipError_t launch_kv_gather(int dtype, bool fp8, const KVView& c, void* k, int64_t ldk, void* v, int64_t ldv, hipStream_t s)
{
    const int esz = dtype == MOE_BF16 ? 2 : 4;
    if (!fp8)
        return by_lanes(c, c.D * esz / 16, [&](auto lpr, unsigned blocks) {
            constexpr int L = decltype(lpr)::value;
            gather_kernel<L><<<blocks, 256, 0, s>>>(c, static_cast<char*>(k), ldk, static_cast<char*>(v), ldv, esz);
            return hipGetLastError();
        });
    return by_lanes(c, c.D / 8, [&](auto lpr, unsigned blocks) {
        constexpr int L = decltype(lpr)::value;
        if (dtype == MOE_BF16)
            gather_fp8_kernel<bf16_t, L><<<blocks, 256, 0, s>>>(c, static_cast<bf16_t*>(k), ldk, static_cast<bf16_t*>(v), ldv);
        else
            gather_fp8_kernel<float, L><<<blocks, 256, 0, s>>>(c, static_cast<float*>(k), ldk, static_cast<float*>(v), ldv);
        return hipGetLastError();
    });
}

}  // namespace moe
