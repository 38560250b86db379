// Which tokens of a sequence and head to keep: those of the largest keys, by a radix selection, listed in order.
//
// Key of a token: 0 where it is not there; the largest for the first and the recent ones; between them its score, as an integer that orders like it.
// Three counts of 11, 11 and 10 bits, from the top, find the key T that the last kept token has, and how many of those equal to T are kept;
// ranks among the larger keys and the first so many equal ones are then the places in the list.
//
// A block has a sequence and head, 4 consecutive tokens of every 4096 to a thread: up to 49152 tokens are read once and stay in registers.  What bounds it:
// latency and barriers for short sequences (32 of up to 4096 tokens in 8 heads, a block to a unit: 8.5 us); for longer ones their loads, each in a branch of its own and waited for
// there, and the counting in LDS (32 of 16000 tokens 21 us, 20000 38, 45000 49; of 60000, read for every count, 107).
//
// Where few sequences are long, one to a unit leaves most of the chip idle: their tokens are cut into parts, a block each, and three launches follow each
// other: counts of the first 11 bits; the keys of the bin that holds T, written down; T from those, and the list.  (Kernel boundaries are the waits; every block
// finds T for itself.)  Two sequences of 131072 tokens in 4 heads: 26 us, launches of 5, 8 and 13 us, chains of barriers and of loads as above; 153 with a block to each
// sequence and head, 385 as four counts of 8 bits that read the scores every time.
#include "kv.h"

namespace moe {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2048, kCopies = 4;      // lanes count in four copies: equal digits of a wave meet a quarter as often

struct Shared {
    uint32_t hist[kBins * kCopies];
    uint32_t sums[kWaves], found[4];
    uint32_t above[16 * kWaves], same[16 * kWaves];      // of the groups of 256 tokens that a wave has at a time
};

struct Sequence {
    int s, h, kv, held;
};

// The keys of tokens j .. j + 3 (a multiple of 4: they share a page).
struct Four {
    uint32_t k[4];
};
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x == 0.0f ? 0.0f : x);       // (both zeros are the same)
    const uint32_t k = (u >> 31) ? ~u : u | 0x80000000u;            // minus infinity 0x7fffff, infinity 0xff800000
    return x != x || k == 0x007fffffu ? 1u : k;
}
__device__ __forceinline__ int page_id(const SelectArgs& a, const Sequence& q, int j)
{
    return j < q.held ? a.c.table[(int64_t)q.s * a.c.max_pages + (j >> a.c.page_shift)] : -1;
}
__device__ __forceinline__ Four keys_of(const SelectArgs& a, const Sequence& q, int j, int id)
{
    Four f{{0, 0, 0, 0}};
    if (id < 0 || id >= a.c.n_pages) return f;
    const float4 x = *reinterpret_cast<const float4*>(a.scores + page_row(id, a.c.Hk, q.h, a.c.page_shift, j & ((1 << a.c.page_shift) - 1)));
    const float v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = j + i;
        f.k[i] = t >= q.held ? 0 : t < a.first || t >= q.kv - a.recent ? 0xffffffffu : key_of(v[i]);
    }
    return f;
}

// The bin in which the rank-th key from the top lies, and its rank in the bin, as found[0] and found[1] (if there are so many), from the counts of
// bins kBins - 1 - 2 tid and one below; returns their sum.  Every thread calls it.
__device__ __forceinline__ uint32_t find_bin(Shared& sh, const uint32_t (&n)[2], uint32_t rank)
{
    const int tid = threadIdx.x, wave = tid >> 6;
    uint32_t incl = (uint32_t)wave_scan((int)(n[0] + n[1]));
    if (lane_id() == 63) sh.sums[wave] = incl;
    __syncthreads();
    uint32_t total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const uint32_t v = sh.sums[w];
        incl += w < wave ? v : 0;
        total += v;
    }
    const uint32_t before = incl - n[0] - n[1];
    if (before < rank && rank <= incl) {
        const bool first = rank <= before + n[0];
        sh.found[0] = (uint32_t)(kBins - 1 - 2 * tid - (first ? 0 : 1));
        sh.found[1] = rank - before - (first ? 0 : n[0]);
    }
    __syncthreads();
    return total;
}

// The search for T.  each_key: calls a function with all keys of the sequence.
struct Threshold {
    uint32_t key, equal;      // T, and how many tokens of this key are kept
    int kept;                 // tokens that are kept; all that are there if `all`
    bool all;
};
// FIRST: of its counts; with 1, `prefix` has the digit of the first and `rank` is that in its bin.
template <int FIRST, typename F> __device__ __forceinline__ Threshold find_threshold(Shared& sh, uint32_t prefix, uint32_t rank, F each_key)
{
    const int tid = threadIdx.x, lane = lane_id();
    Threshold t{0, 0, 0, false};
#pragma unroll 1
    for (int pass = FIRST; pass < 3; ++pass) {
        const int bits = pass < 2 ? 11 : 10, shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        uint4* clear = reinterpret_cast<uint4*>(sh.hist);
        for (int i = tid; i < kBins * kCopies / 4; i += kThreads) clear[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        const uint32_t want = pass == 0 ? 0 : prefix >> (shift + bits);
        each_key([&](uint32_t k) {
            if (k != 0 && (pass == 0 || (k >> (shift + bits)) == want)) atomicAdd(&sh.hist[((k >> shift) & ((1u << bits) - 1)) * kCopies + (lane & (kCopies - 1))], 1u);
        });
        __syncthreads();
        // bins from the top, two to a thread
        uint32_t n[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4 v = clear[kBins - 1 - 2 * tid - i];
            n[i] = (v.x + v.y) + (v.z + v.w);
        }
        const uint32_t total = find_bin(sh, n, rank);
        if (pass == 0) {
            t.kept = total < rank ? (int)total : (int)rank;
            t.all = total <= rank;
            if (t.all) return t;
        }
        prefix |= sh.found[0] << shift;
        rank = sh.found[1];
    }
    t.key = prefix;
    t.equal = rank;
    return t;
}

// Lists the kept tokens of up to 4096 N tokens from j0 on; kept, equal: larger and equal keys before them.
template <int N> __device__ __forceinline__ void list_tokens(const SelectArgs& a, Shared& sh, const Threshold& t, const Four (&f)[N], int j0, int32_t* keep,
                                                             uint32_t& kept, uint32_t& equal)
{
    const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
    auto over = [&](uint32_t k) { return k != 0 && (t.all || k > t.key); };
    auto same = [&](uint32_t k) { return !t.all && k == t.key; };
#pragma unroll
    for (int i = 0; i < N; ++i) {
        uint32_t o = 0, e = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            o += __popcll(__ballot(over(f[i].k[c])));
            e += __popcll(__ballot(same(f[i].k[c])));
        }
        if (lane == 0) {
            sh.above[i * kWaves + wave] = o;
            sh.same[i * kWaves + wave] = e;
        }
    }
    __syncthreads();
    // sums over the groups, in their order: a wave's lanes take N each
    uint32_t all_o, all_e;
    {
        const int lanes = 16 * N;
        uint32_t o[(16 * N + 63) / 64], e[(16 * N + 63) / 64];
        constexpr int PER = (16 * N + 63) / 64;
        uint32_t so = 0, se = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int at = lane * PER + i;
            o[i] = at < lanes ? sh.above[at] : 0;
            e[i] = at < lanes ? sh.same[at] : 0;
            so += o[i];
            se += e[i];
        }
        uint32_t io = (uint32_t)wave_scan((int)so), ie = (uint32_t)wave_scan((int)se);
        all_o = (uint32_t)__builtin_amdgcn_readlane((int)io, 63);
        all_e = (uint32_t)__builtin_amdgcn_readlane((int)ie, 63);
        io -= so;
        ie -= se;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int at = lane * PER + i;
                if (at < lanes) {
                    sh.above[at] = io;
                    sh.same[at] = ie;
                }
                io += o[i];
                ie += e[i];
            }
        }
        __syncthreads();
    }
    const unsigned long long under = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        uint32_t o = kept + sh.above[i * kWaves + wave], e = equal + sh.same[i * kWaves + wave];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            o += __popcll(__ballot(over(f[i].k[c])) & under);
            e += __popcll(__ballot(same(f[i].k[c])) & under);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const bool is_over = over(f[i].k[c]), is_same = same(f[i].k[c]);
            const uint32_t at = o + (e < t.equal ? e : t.equal);
            if ((is_over || (is_same && e < t.equal)) && at < (uint32_t)a.budget) keep[at] = j0 + i * 4 * kThreads + tid * 4 + c;
            o += is_over;
            e += is_same;
        }
    }
    kept += all_o;
    equal += all_e;
}

template <int N> __device__ __forceinline__ void read_keys(const SelectArgs& a, const Sequence& q, int j0, Four (&f)[N])
{
    constexpr int AT_ONCE = N < 8 ? N : 8;      // (12 are eight and four)
#pragma unroll
    for (int i0 = 0; i0 < N; i0 += AT_ONCE) {
        const int n = N - i0 < AT_ONCE ? N - i0 : AT_ONCE;
        int id[AT_ONCE];
#pragma unroll
        for (int i = 0; i < n; ++i) id[i] = page_id(a, q, j0 + (i0 + i) * 4 * kThreads + (int)threadIdx.x * 4);
#pragma unroll
        for (int i = 0; i < n; ++i) f[i0 + i] = keys_of(a, q, j0 + (i0 + i) * 4 * kThreads + (int)threadIdx.x * 4, id[i]);
        if (i0 + AT_ONCE < N) __builtin_amdgcn_sched_barrier(0);
    }
}

// A sequence that 4096 N tokens hold, its keys in registers.
template <int N> __device__ __forceinline__ int select_held(const SelectArgs& a, const Sequence& q, Shared& sh, int32_t* keep)
{
    Four f[N];
    read_keys(a, q, 0, f);
    const Threshold t = find_threshold<0>(sh, 0, (uint32_t)a.budget, [&](auto count) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) count(f[i].k[c]);
    });
    uint32_t kept = 0, equal = 0;
    list_tokens(a, sh, t, f, 0, keep, kept, equal);
    return t.kept;
}
// A longer one: read again for every count.
__device__ __forceinline__ int select_long(const SelectArgs& a, const Sequence& q, Shared& sh, int32_t* keep)
{
    constexpr int N = 8;
    const Threshold t = find_threshold<0>(sh, 0, (uint32_t)a.budget, [&](auto count) {
#pragma unroll 1
        for (int j = 0; j < q.held; j += N * 4 * kThreads) {
            Four f[N];
            read_keys(a, q, j, f);
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) count(f[i].k[c]);
        }
    });
    uint32_t kept = 0, equal = 0;
#pragma unroll 1
    for (int j = 0; j < q.held; j += N * 4 * kThreads) {
        Four f[N];
        read_keys(a, q, j, f);
        list_tokens(a, sh, t, f, j, keep, kept, equal);
        __syncthreads();
    }
    return t.kept;
}

__device__ __forceinline__ Sequence sequence_of(const SelectArgs& a)
{
    Sequence q;
    q.s = blockIdx.x / a.c.Hk;
    q.h = blockIdx.x - q.s * a.c.Hk;
    q.kv = a.c.lens[q.s] > 0 ? a.c.lens[q.s] : 0;
    const int most = a.c.max_pages << a.c.page_shift;
    q.held = q.kv < most ? q.kv : most;
    return q;
}

__device__ __forceinline__ void finish(const SelectArgs& a, const Sequence& q, int32_t* keep, int m, int first, int step)
{
    if (q.h == 0 && first == 0) a.keep_lens[q.s] = m;
    for (int64_t i = (int64_t)m + first; i < a.budget; i += step) keep[i] = -1;
}

// A sequence and head to a block.
__device__ __forceinline__ void select_alone(const SelectArgs& a, const Sequence& q, Shared& sh)
{
    int32_t* keep = a.keep + (int64_t)blockIdx.x * a.budget;
    int m;
    if (q.held <= 4 * kThreads) m = select_held<1>(a, q, sh, keep);
    else if (q.held <= 16 * kThreads) m = select_held<4>(a, q, sh, keep);
    else if (q.held <= 48 * kThreads) m = select_held<12>(a, q, sh, keep);      // (16 would spill)
    else m = select_long(a, q, sh, keep);
    finish(a, q, keep, m, threadIdx.x, kThreads);
}
__global__ __launch_bounds__(kThreads) void select_kernel(SelectArgs a)
{
    __shared__ __attribute__((aligned(16))) Shared sh;
    select_alone(a, sequence_of(a), sh);
}

// ---- sequences in parts: blockIdx.y of them, of whole fours of tokens ----
constexpr int kPartTokens = 2 * 4 * kThreads, kMaxParts = 2 * kWaves;
struct Parts {
    uint32_t* counts;      // [sequence and head][part][kBins], of the keys' first digits
    uint32_t* keys;        // [sequence and head][tokens]: in a part's place the keys of the bin that holds T
    uint32_t* sizes;       // [sequence and head][part][2]: how many of these, and how many larger keys
    int64_t tokens;
};
struct Part {
    int per, begin, end, used;      // tokens of a part, this one's, parts that have some
};
__device__ __forceinline__ Part part_of(const Sequence& q)
{
    Part p;
    p.per = ((q.held + (int)gridDim.y - 1) / (int)gridDim.y + 3) & ~3;
    if (p.per < kPartTokens) p.per = kPartTokens;
    p.used = (q.held + p.per - 1) / p.per;
    const int64_t begin = (int64_t)blockIdx.y * p.per;
    p.begin = begin < q.held ? (int)begin : q.held;
    p.end = q.held - p.begin < p.per ? q.held : p.begin + p.per;
    return p;
}
// Up to this length a block does it alone, in the first launch.
constexpr int kAlone = 4 * 4 * kThreads;

// The keys of a part, 8 of a thread at a time: f(keys, the first token of the block's).
template <typename F> __device__ __forceinline__ void part_keys(const SelectArgs& a, Sequence q, const Part& p, F f)
{
    q.held = p.end;
#pragma unroll 1
    for (int j = p.begin; j < p.end; j += kPartTokens) {
        Four k[2];
        read_keys(a, q, j, k);
        f(k, j);
    }
}

__global__ __launch_bounds__(kThreads) void count_parts_kernel(SelectArgs a, Parts w)
{
    __shared__ __attribute__((aligned(16))) Shared sh;
    const Sequence q = sequence_of(a);
    if (q.held <= kAlone) {
        if (blockIdx.y == 0) select_alone(a, q, sh);
        return;
    }
    const Part p = part_of(q);
    if ((int)blockIdx.y >= p.used) return;
    const int tid = threadIdx.x, lane = lane_id();
    uint4* clear = reinterpret_cast<uint4*>(sh.hist);
    for (int i = tid; i < kBins * kCopies / 4; i += kThreads) clear[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    part_keys(a, q, p, [&](const Four (&k)[2], int) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t key = k[i / 4].k[i % 4];
            if (key != 0) atomicAdd(&sh.hist[(key >> 21) * kCopies + (lane & (kCopies - 1))], 1u);
        }
    });
    __syncthreads();
    uint32_t* counts = w.counts + ((int64_t)blockIdx.x * gridDim.y + blockIdx.y) * kBins;
    for (int i = tid; i < kBins; i += kThreads) {
        const uint4 v = clear[i];
        counts[i] = (v.x + v.y) + (v.z + v.w);
    }
}

// The bin that holds T, from all parts' counts.
__device__ __forceinline__ uint32_t bin_of_parts(const SelectArgs& a, const Parts& w, const Part& p, Shared& sh)
{
    uint32_t n[2] = {0, 0};
    const uint32_t* counts = w.counts + (int64_t)blockIdx.x * gridDim.y * kBins + (kBins - 2 - 2 * threadIdx.x);
#pragma unroll 8
    for (int i = 0; i < p.used; ++i) {
        const uint2 v = *reinterpret_cast<const uint2*>(counts + (int64_t)i * kBins);
        n[0] += v.y;
        n[1] += v.x;
    }
    return find_bin(sh, n, (uint32_t)a.budget);
}

__global__ __launch_bounds__(kThreads) void gather_parts_kernel(SelectArgs a, Parts w)
{
    __shared__ __attribute__((aligned(16))) Shared sh;
    const Sequence q = sequence_of(a);
    const Part p = part_of(q);
    if (q.held <= kAlone || (int)blockIdx.y >= p.used) return;
    const uint32_t total = bin_of_parts(a, w, p, sh);
    if (total <= (uint32_t)a.budget) return;
    const uint32_t bin = sh.found[0];
    __syncthreads();
    if (threadIdx.x < 2) sh.found[threadIdx.x] = 0;
    __syncthreads();
    uint32_t* keys = w.keys + (int64_t)blockIdx.x * w.tokens + p.begin;
    const int lane = lane_id();
    uint32_t larger = 0;
    part_keys(a, q, p, [&](const Four (&k)[2], int) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t key = k[i / 4].k[i % 4];
            const unsigned long long mine = __ballot(key != 0 && (key >> 21) == bin);
            larger += __popcll(__ballot(key != 0 && (key >> 21) > bin));
            uint32_t at = 0;
            if (mine != 0) {      // (in any order: they are only counted)
                if (lane == 0) at = atomicAdd(&sh.found[0], (uint32_t)__popcll(mine));
                at = (uint32_t)__builtin_amdgcn_readfirstlane((int)at) + __popcll(mine & ((1ull << lane) - 1));
                if ((mine >> lane) & 1) keys[at] = key;
            }
        }
    });
    if (lane == 0) atomicAdd(&sh.found[1], larger);
    __syncthreads();
    if (threadIdx.x < 2) w.sizes[((int64_t)blockIdx.x * gridDim.y + blockIdx.y) * 2 + threadIdx.x] = sh.found[threadIdx.x];
}

__global__ __launch_bounds__(kThreads) void list_parts_kernel(SelectArgs a, Parts w)
{
    __shared__ __attribute__((aligned(16))) Shared sh;
    __shared__ uint32_t over[kMaxParts], same[kMaxParts];
    const Sequence q = sequence_of(a);
    const Part p = part_of(q);
    if (q.held <= kAlone || (int)blockIdx.y >= p.used) return;
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    const uint32_t total = bin_of_parts(a, w, p, sh);
    Threshold t{0, 0, (int)total, true};
    // a wave has the keys of parts `wave` and `wave` + 16
    auto keys_of_part = [&](int part, auto f) {
        const uint32_t n = w.sizes[((int64_t)blockIdx.x * gridDim.y + part) * 2];
        const uint32_t* keys = w.keys + (int64_t)blockIdx.x * w.tokens + (int64_t)part * p.per;
#pragma unroll 4
        for (uint32_t i = lane; i < n; i += 64) f(keys[i]);
    };
    uint32_t kept = 0, equal = 0;
    if (total > (uint32_t)a.budget) {
        const uint32_t bin = sh.found[0], rank = sh.found[1];
        t = find_threshold<1>(sh, bin << 21, rank, [&](auto count) {
            for (int part = wave; part < p.used; part += kWaves) keys_of_part(part, count);
        });
        t.kept = a.budget;
        // what is kept of the parts before this one
        for (int part = wave; part < p.used; part += kWaves) {
            uint32_t o = 0, e = 0;
            if (part < (int)blockIdx.y) {
                keys_of_part(part, [&](uint32_t k) {
                    o += k > t.key;
                    e += k == t.key;
                });
            }
            o = (uint32_t)wave_scan((int)o);
            e = (uint32_t)wave_scan((int)e);
            if (lane == 63) {
                over[part] = o + (part < (int)blockIdx.y ? w.sizes[((int64_t)blockIdx.x * gridDim.y + part) * 2 + 1] : 0);
                same[part] = e;
            }
        }
        __syncthreads();
        for (int part = 0; part < (int)blockIdx.y; ++part) {
            kept += over[part];
            equal += same[part];
        }
    } else {
        // all of them: count what is there before (tables with holes)
        if (threadIdx.x == 0) sh.found[0] = 0;
        __syncthreads();
        uint32_t n = 0;
        for (int part = 0; part < (int)blockIdx.y; ++part) {
            const uint2 v = reinterpret_cast<const uint2*>(w.counts + ((int64_t)blockIdx.x * gridDim.y + part) * kBins)[threadIdx.x];
            n += v.x + v.y;
        }
        n = (uint32_t)wave_scan((int)n);
        if (lane == 63) atomicAdd(&sh.found[0], n);
        __syncthreads();
        kept = sh.found[0];
    }
    int32_t* keep = a.keep + (int64_t)blockIdx.x * a.budget;
    part_keys(a, q, p, [&](const Four (&k)[2], int j) {
        list_tokens(a, sh, t, k, j, keep, kept, equal);
        __syncthreads();
    });
    finish(a, q, keep, t.kept, blockIdx.y * kThreads + threadIdx.x, p.used * kThreads);
}

}  // namespace

hipError_t launch_kv_select(const SelectArgs& a, void* workspace, size_t bytes, hipStream_t s)
{
    const int64_t items = (int64_t)a.c.S * a.c.Hk, longest = (int64_t)a.c.max_pages << a.c.page_shift;
    if (items > kMaxBlocks / 4) return hipErrorInvalidConfiguration;      // (of four times 256 threads)
    int units = 0;
    const hipError_t e = compute_units(&units);
    if (e != hipSuccess) return e;
    if (items < units && longest > kAlone) {
        int64_t parts = (longest + kPartTokens - 1) / kPartTokens, most = 4 * (int64_t)units / items;
        most = most < 2 ? 2 : most > kMaxParts ? kMaxParts : most;
        parts = parts < most ? parts : most;
        Parts w;
        w.tokens = longest;
        w.counts = static_cast<uint32_t*>(workspace);
        w.sizes = w.counts + items * parts * kBins;
        w.keys = w.sizes + items * parts * 2;
        if ((size_t)((items * parts * (kBins + 2) + items * longest) * 4) <= bytes) {
            const dim3 grid((unsigned)items, (unsigned)parts);
            count_parts_kernel<<<grid, kThreads, 0, s>>>(a, w);
            gather_parts_kernel<<<grid, kThreads, 0, s>>>(a, w);
            list_parts_kernel<<<grid, kThreads, 0, s>>>(a, w);
            return hipGetLastError();
        }
    }
    select_kernel<<<(unsigned)items, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace moe
