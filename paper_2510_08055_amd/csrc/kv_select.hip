// Which tokens of a sequence and head to keep: those of the largest keys, by a radix selection, listed in order.
//
// Key of a token: 0 where it is not there; the largest for the first and the recent ones; between them its score, as an integer that orders like it.
#include "kv.h"

namespace moe {
namespace {

constexpr int kThreads = 1024;

__device__ __forceinline__ uint32_t key_of(const SelectArgs& a, int s, int h, int j, int kv)
{
    const KVView& c = a.c;
    const int id = c.table[(int64_t)s * c.max_pages + (j >> c.page_shift)];
    if (id < 0 || id >= c.n_pages) return 0;
    if (j < a.first || j >= kv - a.recent) return 0xffffffffu;
    const float x = a.scores[page_row(id, c.Hk, h, c.page_shift, j & ((1 << c.page_shift) - 1))];
    if (x != x) return 1;
    const uint32_t u = __float_as_uint(x == 0.0f ? 0.0f : x);       // (both zeros are the same)
    const uint32_t k = (u >> 31) ? ~u : u | 0x80000000u;            // minus infinity 0x7fffff, infinity 0xff800000
    return k == 0x007fffffu ? 1 : k;
}

__global__ __launch_bounds__(kThreads) void select_kernel(SelectArgs a)
{
    const KVView& c = a.c;
    __shared__ uint32_t hist[256], sums[2][kThreads / 64], found[2];
    const int s = blockIdx.x / c.Hk, h = blockIdx.x - s * c.Hk;
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    const int kv = c.lens[s] > 0 ? c.lens[s] : 0;
    const int most = c.max_pages << c.page_shift, held = kv < most ? kv : most;
    int32_t* keep = a.keep + (int64_t)blockIdx.x * a.budget;

    // digits from the top: the key of which `rank` or fewer tokens have a larger one
    uint32_t prefix = 0, rank = (uint32_t)a.budget;
    int there = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (threadIdx.x < 256) hist[threadIdx.x] = 0;
        __syncthreads();
        for (int j = threadIdx.x; j < held; j += kThreads) {
            const uint32_t k = key_of(a, s, h, j, kv);
            if (k != 0 && (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8)))) atomicAdd(&hist[(k >> shift) & 255], 1u);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            uint32_t above = 0;
            int d = 255;
            for (; d > 0 && above + hist[d] < rank; --d) above += hist[d];
            found[0] = prefix | (uint32_t)d << shift;
            found[1] = rank - above;
            if (shift == 24) {
                uint32_t all = 0;
                for (int i = 0; i < 256; ++i) all += hist[i];
                sums[0][0] = all;
            }
        }
        __syncthreads();
        prefix = found[0];
        rank = found[1];
        if (shift == 24) there = (int)sums[0][0];
        __syncthreads();
        if (there <= a.budget) break;
    }
    const bool all = there <= a.budget;
    const int m = all ? there : a.budget;
    if (h == 0 && threadIdx.x == 0) a.keep_lens[s] = m;
    // in order: keys above, and the first `rank` of those equal
    uint32_t kept = 0, equal = 0;
    for (int j0 = 0; j0 < held; j0 += kThreads) {
        const int j = j0 + threadIdx.x;
        const uint32_t k = j < held ? key_of(a, s, h, j, kv) : 0;
        const bool over = k != 0 && (all || k > prefix), same = k != 0 && !all && k == prefix;
        const unsigned long long b0 = __ballot(over), b1 = __ballot(same), under = (1ull << lane) - 1;
        if (lane == 0) {
            sums[0][wave] = __popcll(b0);
            sums[1][wave] = __popcll(b1);
        }
        __syncthreads();
        uint32_t o = kept, e = equal, o_all = 0, e_all = 0;
        for (int w = 0; w < kThreads / 64; ++w) {
            if (w < wave) {
                o += sums[0][w];
                e += sums[1][w];
            }
            o_all += sums[0][w];
            e_all += sums[1][w];
        }
        o += __popcll(b0 & under);
        e += __popcll(b1 & under);
        const uint32_t at = o + (e < rank ? e : rank);
        if ((over || (same && e < rank)) && at < (uint32_t)a.budget) keep[at] = j;
        kept += o_all;
        equal += e_all;
        __syncthreads();
    }
    for (int i = m + threadIdx.x; i < a.budget; i += kThreads) keep[i] = -1;
}

}  // namespace

hipError_t launch_kv_select(const SelectArgs& a, hipStream_t s)
{
    const int64_t blocks = (int64_t)a.c.S * a.c.Hk;
    if (blocks > kMaxBlocks / 4) return hipErrorInvalidConfiguration;      // (of four times 256 threads)
    select_kernel<<<(unsigned)blocks, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace moe
