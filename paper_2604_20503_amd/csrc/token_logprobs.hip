// Log probabilities of given tokens, the entropy and the largest alternatives of rows of logits.
//     x_v = (z_v - m) / T with m the row's largest logit,  S = sum_v exp x_v
//     log p_v = x_v - log S,   H = log S - sum_v exp(x_v) x_v / S
// Differences are taken before they are scaled, so that logits of any size keep their digits; H is a sum of terms of one sign.
//
// One pass over the logits: a row is cut into chunks, a workgroup takes a chunk tile by tile, a thread a *group* of 32 bytes of each
// tile.  Beside its running (m, S, sum) it leaves the largest logit of every group in LDS, and nothing else is done for the
// alternatives while the logits go by.  The K largest of a chunk lie in the K groups whose largest logits come first: with
// keys (logit, lowest id) any K groups that come before a group hold K logits that come before all of that group's.  Those groups are
// found in LDS and read once more, 32 K bytes.  The workgroup of a row that is done last joins the chunks.
//
// 400 rows of 152064 fp32 logits with 20 alternatives (243 MB): 54.6 us, 4.5 TB/s (a copy of 1 GiB: 5.1); the rest is the tail of each
// workgroup, its alternatives and the join.  5 rows of 128256 bf16 logits: 9.6 us, in which a chunk's tiles, its ranking and the join follow
// each other.
#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "common.hpp"
#include "device_utils.hpp"

namespace fsr {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453094;

struct LogprobArgs {
    const void* logits;
    const int32_t* n_rows;
    const int32_t* tokens;
    float* logprobs;
    float* entropy;
    int32_t* top_ids;
    float* top_logprobs;
    long long stride;
    int N_cap, V, M, K;
    float scale;   // log2(e) / T
    double inv_t;
    int chunks, tiles;  // of a row, of a chunk
    unsigned long long* arrivals;  // [N_cap], kArrivalStep apart
    uint64_t* stats;    // [N_cap * chunks][3]: m, S, sum of S's terms times x, as doubles
    uint64_t* keys;     // [N_cap * chunks][K]
    unsigned long long call_id;
};

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

// What another workgroup of the launch reads: stored through to memory, loaded past the caches.
__device__ __forceinline__ void publish(uint64_t* p, uint64_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint64_t fetch(const uint64_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__device__ __forceinline__ float value_of(const float* p) { return *p; }
__device__ __forceinline__ float value_of(const uint16_t* p) { return __builtin_bit_cast(float, (uint32_t)*p << 16); }

// Logits in descending order, the lower id first among equals: larger keys come first.  NaN counts as -inf, -0 as 0.
__device__ __forceinline__ uint64_t key_of(float z, int id) {
    if (z != z) z = -INFINITY;
    const uint32_t b = __builtin_bit_cast(uint32_t, z + 0.0f);
    return (uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (uint32_t)~id;
}
__device__ __forceinline__ float value_of_key(uint64_t key) {
    const uint32_t b = (uint32_t)(key >> 32);
    return __builtin_bit_cast(float, b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ int id_of_key(uint64_t key) { return (int)~(uint32_t)key; }

constexpr int kTilesMax = 32;    // of a chunk
constexpr int kChunksMax = 64;   // of a row
constexpr int kWorkgroups = 1024; // that a call is cut into, if its rows are fewer
constexpr int kArrivalStep = 16;  // words from a row's arrival counter to the next: a line of memory each (side by side: 64 rows of 32 chunks 56 us)
constexpr int kGroupsMax = 512;  // groups that may hold alternatives, listed
constexpr int kGroupsMore = 32;   // than K, that are read as they are
constexpr float kLeast = -200.0f; // least power of two that is told from no weight at all
static_assert((long long)kTilesMax * kChunksMax * kThreads * 8 == 1 << 22, "longest row of fp32");

// Eight or sixteen logits: 32 bytes.
template <typename T>
struct Group;
template <>
struct Group<float> {
    static constexpr int kN = 8;
    f32x4 a, b;
    __device__ __forceinline__ void load(const float* p) { __builtin_memcpy(&a, p, 16); __builtin_memcpy(&b, p + 4, 16); }
    __device__ __forceinline__ float get(int k) const { return k < 4 ? a[k] : b[k - 4]; }
};
template <>
struct Group<uint16_t> {
    static constexpr int kN = 16;
    u32x4 a, b;
    __device__ __forceinline__ void load(const uint16_t* p) { __builtin_memcpy(&a, p, 16); __builtin_memcpy(&b, p + 8, 16); }
    __device__ __forceinline__ float get(int k) const {
        const uint32_t w = k < 8 ? a[k >> 1] : b[(k - 8) >> 1];
        return __builtin_bit_cast(float, k & 1 ? w & 0xffff0000u : w << 16);
    }
};

// Sums of weights 2^x and of weights times x, x = (z - m) * scale.
struct Sums {
    float m, s, e;
    // Refers them to a larger logit.
    __device__ __forceinline__ void refer(float to, float scale) {
        const float d = fmaxf((m - to) * scale, kLeast), w = __builtin_amdgcn_exp2f(d);
        e = fmaf(d, s, e) * w;
        s *= w;
        m = to;
    }
    template <int N, class Get>
    __device__ __forceinline__ void add(Get get, float top, float scale) {
        if (__any(top > m)) {
            if (top > m) refer(top, scale);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float x = fmaxf((get(k) - m) * scale, kLeast);  // (NaN, -inf: no weight)
            const float w = __builtin_amdgcn_exp2f(x);
            s += w;
            e = fmaf(w, x, e);
        }
    }
};

// Steps of a reduction over the wave by DPP: lanes 1, 2, 4, 8 to the left in a row of 16, then lane 15 of a row to the next one, lane 31
// to the upper half; lane 63 has it all.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_max(float v) {
    return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false)));
}
__device__ __forceinline__ float wave_max_by_dpp(float v) {
    v = dpp_max<0x111, 0xf>(v);
    v = dpp_max<0x112, 0xf>(v);
    v = dpp_max<0x114, 0xf>(v);
    v = dpp_max<0x118, 0xf>(v);
    v = dpp_max<0x142, 0xa>(v);
    v = dpp_max<0x143, 0xc>(v);
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), kWave - 1));
}
__device__ __forceinline__ uint32_t wave_largest(uint32_t v) {
    auto step = [&](auto ctrl, auto rows) {
        const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        v = other > v ? other : v;
    };
    step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
    return (uint32_t)__builtin_amdgcn_readlane((int)v, kWave - 1);
}
// The larger key of a lane and its neighbour in a group of four.
template <int PERM>
__device__ __forceinline__ uint64_t larger_of_four(uint64_t k) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)k, PERM, 0xf, 0xf, true), hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(k >> 32), PERM, 0xf, 0xf, true);
    const uint64_t other = (uint64_t)hi << 32 | lo;
    return other > k ? other : k;
}

struct Shared {
    double s[kThreads / kWave], e[kThreads / kWave], more;
    float m[kThreads / kWave];
    uint32_t set_top[kWave], set_id[kWave];  // keys of 64 sets, in halves
    // Lengths of the lists: of groups, of the chunk's keys, of all chunks' keys.  Each has a counter of its own, cleared at the start: one that is
    // used again would have to be cleared behind a barrier that every wave reaches after it has read it.
    int groups, keys, joined;
    int count[kThreads / kWave], last;
    uint64_t top[FSR_TOP_MAX];
    uint64_t list[kGroupsMax];
};

// The K largest of n keys (all different, or 0: none), in descending order; 0 behind the last one.  Called by the whole workgroup, whose
// keys are in LDS behind a barrier; top is there behind the next one.
__device__ __forceinline__ void rank(const uint64_t* keys, int n, int K, uint64_t* top) {
    for (int k = threadIdx.x; k < K; k += kThreads) top[k] = 0;
    __syncthreads();
    for (int c = threadIdx.x; c < n; c += kThreads) {
        const uint64_t mine = keys[c];
        int before = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) before += keys[j] > mine;
        if (mine != 0 && before < K) top[before] = mine;
    }
}

// A key that r of 64 keys in LDS (all different, or 0: none) are not below, and few others; 1 if there are not so many.  By every wave
// for itself.  Their upper halves alone are compared, unless many of them are equal.
__device__ __forceinline__ uint64_t rth_of_64(const Shared& sh, int r) {
    const int lane = threadIdx.x & (kWave - 1);
    const uint32_t top = sh.set_top[lane];
    int before = 0;
#pragma unroll
    for (int j = 0; j < kWave; ++j) before += sh.set_top[j] > top;
    // the r-th largest upper half, some lane's that has it: fewer than r are larger, and with its equals there are r
    uint32_t bound = before < r ? top : 0xffffffffu;
    bound = ~(uint32_t)wave_largest(~bound);
    const unsigned long long equal = __ballot(top == bound);
    if (bound == 0) return 1;
    if (__popcll(equal) <= 8) return (uint64_t)bound << 32;
    const uint64_t mine = (uint64_t)top << 32 | sh.set_id[lane];
    before = 0;
#pragma unroll 8
    for (int j = 0; j < kWave; ++j) before += ((uint64_t)sh.set_top[j] << 32 | sh.set_id[j]) > mine;
    const unsigned long long is = __ballot(before == r - 1);
    if (is == 0) return 1;
    const int at = __ffsll(is) - 1;
    return (uint64_t)bound << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, at);
}

// Groups in descending order of their largest logits, the first of them first among equals.
__device__ __forceinline__ uint64_t group_key(float top, int tile) { return key_of(top, tile * kThreads + threadIdx.x); }

template <typename T, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_kernel(LogprobArgs a) {
    typedef Group<T> G;
    constexpr int N = G::kN, kTile = kThreads * N, kWaves = kThreads / kWave, kAtOnce = 4;
    extern __shared__ __align__(16) char room[];  // largest logits of the groups, then keys
    __shared__ Shared sh;
    float* tops = reinterpret_cast<float*>(room);
    uint64_t* keys = reinterpret_cast<uint64_t*>(room);
    const int row = blockIdx.x / a.chunks, chunk = blockIdx.x - row * a.chunks, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (a.n_rows && row >= a.n_rows[0]) return;
    const T* z = (const T*)a.logits + row * a.stride;
    float given = -INFINITY;  // the logit of this thread's given token: it is there when the row is done
    if ((int)threadIdx.x < a.M) {
        const int id = a.tokens[(size_t)row * a.M + threadIdx.x];
        if (id >= 0 && id < a.V) given = value_of(z + id);
    }
    const int first = chunk * a.tiles * kTile, tiles = min(a.tiles, (a.V - first + kTile - 1) / kTile);
    Sums sums{-3.402823466e38f, 0.0f, 0.0f};
    float best = -INFINITY;
    int best_tile = 0;
    bool any = false;
    auto take = [&](int t, int n, auto get) __attribute__((always_inline)) {  // n logits of the group: 0, or the row ends in it
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < N; ++k) top = fmaxf(top, __builtin_canonicalizef(get(k)));  // (a signalling NaN would take the largest one's place)
        sums.add<N>(get, top, a.scale);
        if (TOP) {
            tops[t * kThreads + threadIdx.x] = top;
            if (n > 0 && (!any || top > best)) { best = top; best_tile = t; any = true; }
        }
    };
    const int mine = first + threadIdx.x * N;
    int t = 0;
    const int whole = min(tiles, (a.V - first) / kTile);
    for (; t + kAtOnce <= whole; t += kAtOnce) {
        G g[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) g[k].load(z + mine + (t + k) * kTile);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) take(t + k, N, [&](int i) __attribute__((always_inline)) { return g[k].get(i); });
    }
    for (; t < whole; ++t) {
        G g;
        g.load(z + mine + t * kTile);
        take(t, N, [&](int i) __attribute__((always_inline)) { return g.get(i); });
    }
    if (t < tiles) {  // the row ends in this tile
        const int at = mine + t * kTile, n = min(max(a.V - at, 0), N);
        float v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < n ? value_of(z + at + i) : -INFINITY;
        take(t, n, [&](int i) __attribute__((always_inline)) { return v[i]; });
    }

    // sums of the chunk
    const float wave_m = wave_max_by_dpp(sums.m);
    if (lane == 0) sh.m[wave] = wave_m;
    if (threadIdx.x == 0) sh.groups = sh.keys = sh.joined = 0;
    // A bound that at least K groups are not below, and few more are: the K-th of the largest keys of 64 sets of four threads each.
    if (TOP) {
        static_assert(kWaves == 4, "four lanes a set");
        uint64_t k = any ? key_of(best, best_tile * kThreads + threadIdx.x) : 0;
        k = larger_of_four<0xb1>(k);  // (lanes 1 0 3 2)
        k = larger_of_four<0x4e>(k);  // (lanes 2 3 0 1)
        if ((threadIdx.x & 3) == 0) {
            sh.set_top[threadIdx.x >> 2] = (uint32_t)(k >> 32);
            sh.set_id[threadIdx.x >> 2] = (uint32_t)k;
        }
    }
    __syncthreads();
    float m = sh.m[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, sh.m[w]);
    const bool has_largest = sums.m == m && sums.s >= 1.0f;  // (its weight is in; a thread without a finite logit has the lowest m there is)
    sums.refer(m, a.scale);
    const double ws = wave_sum_to_last((double)sums.s), we = wave_sum_to_last((double)sums.e);
    if (lane == kWave - 1) { sh.s[wave] = ws; sh.e[wave] = we; }
    if (TOP) {
        const uint64_t least = rth_of_64(sh, a.K);
        const float least_top = value_of_key(least);  // (1: NaN)
        auto has = [&](int t) { return first + t * kTile + (int)threadIdx.x * N < a.V; };
        auto look = [&](float top, int t) __attribute__((always_inline)) {
            if (!(top < least_top) && has(t)) {
                const uint64_t k = group_key(top, t);
                if (k >= least) {
                    const int at = atomicAdd(&sh.groups, 1);
                    if (at < kGroupsMax) sh.list[at] = k;
                }
            }
        };
        int t = 0;
        for (; t + 8 <= tiles; t += 8) {
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = tops[(t + k) * kThreads + threadIdx.x];
#pragma unroll
            for (int k = 0; k < 8; ++k) look(x[k], t + k);
        }
        for (; t < tiles; ++t) look(tops[t * kThreads + threadIdx.x], t);
        __syncthreads();
        int n = sh.groups;
        if (n > kGroupsMax) {
            // Many groups of few threads: the K-th key, bit by bit.
            uint64_t kth = 0;
            for (int bit = 63; bit >= 0; --bit) {
                const uint64_t probe = kth | 1ull << bit;
                int c = 0;
                for (int t = 0; t < tiles; ++t) c += has(t) && group_key(tops[t * kThreads + threadIdx.x], t) >= probe;
                c = wave_sum_i(c);
                if (lane == 0) sh.count[wave] = c;
                __syncthreads();
                c = 0;
                for (int w = 0; w < kWaves; ++w) c += sh.count[w];
                if (c >= a.K) kth = probe;
                __syncthreads();
            }
            if (threadIdx.x == 0) sh.groups = 0;  // (everyone has read it, 64 times two barriers ago)
            __syncthreads();
            for (int t = 0; t < tiles; ++t) {
                const uint64_t k = has(t) ? group_key(tops[t * kThreads + threadIdx.x], t) : 0;
                if (k != 0 && k >= kth) sh.list[min(atomicAdd(&sh.groups, 1), kGroupsMax - 1)] = k;
            }
            __syncthreads();
            n = sh.groups;
        }
        // The logits of those groups that are not below the last group's largest one (of fewer than K groups: all).  A few groups more
        // than K are read as they are.
        const uint64_t* groups_of = sh.list;
        int groups = n;
        uint64_t bound = n < a.K ? 0 : least >> 32 << 32;
        if (n > a.K + kGroupsMore) {
            rank(sh.list, n, a.K, sh.top);
            __syncthreads();
            groups_of = sh.top;
            groups = a.K;
            bound = sh.top[a.K - 1] >> 32 << 32;
        }
        for (int i = threadIdx.x; i < groups * N; i += kThreads) {
            const int id = first + id_of_key(groups_of[i / N]) * N + i % N;
            const uint64_t k = id < a.V ? key_of(value_of(z + id), id) : 0;
            if (k >= bound && k != 0) keys[atomicAdd(&sh.keys, 1)] = k;  // (where the groups' largest logits lay: all have been read)
        }
        __syncthreads();
        n = sh.keys;
        rank(keys, n, a.K, sh.top);
    }
    __syncthreads();
    double S = 0.0, E = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) { S += sh.s[w]; E += sh.e[w]; }
    // A largest logit that has more weight than all others together: log S is small, and those others are its digits.  The thread that met it
    // has added them to a sum of 1 or more, in fp32; its groups are read again, a tile a lane, without the largest logit.  (1000 such rows of 128256
    // bf16 logits: 53.6 us, not 51.0; 5: 10.1, not 9.9.)
    if (S >= 1.0 && S < 2.0) {  // (for the whole workgroup; one logit has the weight 1)
        static_assert(kTilesMax <= kWave, "a tile a lane");
        const unsigned long long holder = __ballot(has_largest);
        if (holder != 0) {
            const int h = __ffsll(holder) - 1, at = first + lane * kTile + (wave * kWave + h) * N;
            float rest = 0.0f;
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float v = lane < tiles && at + k < a.V ? value_of(z + at + k) : m;
                if (v < m) rest += __builtin_amdgcn_exp2f(fmaxf((v - m) * a.scale, kLeast));
            }
            const double sum = wave_sum_to_last((double)rest);
            const float had = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, sums.s), h));
            if (lane == kWave - 1) sh.more = 1.0 - (double)had + sum;
        }
        __syncthreads();
        S += sh.more;
    }

    if (a.chunks > 1) {
        const size_t entry = (size_t)row * a.chunks + chunk;
        if (threadIdx.x == 0) {
            publish(a.stats + 3 * entry, __builtin_bit_cast(uint64_t, (double)m));
            publish(a.stats + 3 * entry + 1, __builtin_bit_cast(uint64_t, S));
            publish(a.stats + 3 * entry + 2, __builtin_bit_cast(uint64_t, E));
        }
        if (TOP)
            for (int k = threadIdx.x; k < a.K; k += kThreads) publish(a.keys + entry * a.K + k, sh.top[k]);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the chunk is in memory once every wave's stores are acknowledged
        __syncthreads();
        if (threadIdx.x == 0) sh.last = count_arrival(a.arrivals + (size_t)row * kArrivalStep, a.call_id) == a.chunks;
        __syncthreads();
        if (!sh.last) return;
        // The chunks' sums, one a lane, in an order that does not depend on who was last (the second wave); their keys beside them, the first
        // 1024 of up to 4096 in registers, and a bound again: of the chunks' j-th keys the r-th, where r chunks with j keys each make K.
        constexpr int kMine = 4;
        const uint64_t* theirs_keys = a.keys + (size_t)row * a.chunks * a.K;
        const int total = a.chunks * a.K;
        uint64_t k[kMine], jth = 0;
        const int nth = TOP ? min((2 * a.K + a.chunks - 1) / a.chunks, a.K) : 1, r = (a.K + nth - 1) / nth;
        if (TOP) {
            if ((int)threadIdx.x < a.chunks) jth = fetch(theirs_keys + threadIdx.x * a.K + nth - 1);
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const int at = threadIdx.x + i * kThreads;
                k[i] = at < total ? fetch(theirs_keys + at) : 0;
            }
        }
        if (wave == 1) {
            const bool in = lane < a.chunks;
            const size_t theirs = (size_t)row * a.chunks + min(lane, a.chunks - 1);
            const double cm = __builtin_bit_cast(double, fetch(a.stats + 3 * theirs)), cs = __builtin_bit_cast(double, fetch(a.stats + 3 * theirs + 1)),
                         ce = __builtin_bit_cast(double, fetch(a.stats + 3 * theirs + 2));
            const float all_m = wave_max_by_dpp(in ? (float)cm : -3.402823466e38f);
            const float d = fmaxf(((float)cm - all_m) * a.scale, kLeast);
            const double w = in ? (double)__builtin_amdgcn_exp2f(d) : 0.0;
            const double all_s = wave_sum_to_last(w * cs), all_e = wave_sum_to_last(w * (ce + (double)d * cs));
            if (lane == kWave - 1) { sh.s[0] = all_s; sh.e[0] = all_e; sh.m[0] = all_m; }
        }
        if (TOP) {
            if (threadIdx.x < kWave) {
                sh.set_top[threadIdx.x] = (uint32_t)(jth >> 32);
                sh.set_id[threadIdx.x] = (uint32_t)jth;
            }
            __syncthreads();
            const uint64_t bound = rth_of_64(sh, r);
            auto list = [&](uint64_t key) { if (key >= bound) keys[atomicAdd(&sh.joined, 1)] = key; };
#pragma unroll
            for (int i = 0; i < kMine; ++i) list(k[i]);
            for (int at = threadIdx.x + kMine * kThreads; at < total; at += kThreads) list(fetch(theirs_keys + at));
            __syncthreads();
            const int n = sh.joined;
            rank(keys, n, a.K, sh.top);
        }
        __syncthreads();
        if (threadIdx.x == 0) __hip_atomic_store(a.arrivals + (size_t)row * kArrivalStep, a.call_id << 16, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for a graph's next replay
        S = sh.s[0];
        E = sh.e[0];
        m = sh.m[0];
    }
    // (No finite logit, or an infinite one: no sum.)  From 2 on the logarithm of S's fraction in fp32 is off by 2^-24 at most, which is less than
    // half a step of a result of .69 and more; below, S - 1 keeps its digits.
    const float sum = (float)S;
    const double log_s = S >= 2.0 ? ((double)__builtin_amdgcn_frexp_expf(sum) + (double)__builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(sum))) * kLn2
                                  : S > 0.0 ? log(S) : __builtin_nan("");
    auto logprob = [&](float zv) { return (float)(((double)zv - (double)m) * a.inv_t - log_s); };
    if (threadIdx.x == 0 && a.entropy) a.entropy[row] = (float)(log_s - E / S * kLn2);
    for (int t = threadIdx.x; t < a.M; t += kThreads) {
        float zv = given;
        if (t >= kThreads) {
            const int id = a.tokens[(size_t)row * a.M + t];
            zv = id >= 0 && id < a.V ? value_of(z + id) : -INFINITY;
        }
        if (zv != zv) zv = -INFINITY;
        a.logprobs[(size_t)row * a.M + t] = logprob(zv);
    }
    if (TOP)
        for (int k = threadIdx.x; k < a.K; k += kThreads) {
            a.top_ids[(size_t)row * a.K + k] = id_of_key(sh.top[k]);
            a.top_logprobs[(size_t)row * a.K + k] = logprob(value_of_key(sh.top[k]));
        }
}

// How a call is cut, and its workspace: arrivals [rows], (m, S, sum) [entries][3], keys [entries][K].
struct Cut {
    int chunks, tiles;  // of a row, of a chunk
    size_t arrivals, stats, keys, total;
};
Cut cut(const fsr_logprob_params* p) {
    const int tile = kThreads * (p->dtype == FSR_F32 ? 8 : 16), all = (p->V + tile - 1) / tile, least = (all + kTilesMax - 1) / kTilesMax;
    const long long n = std::max(p->N_cap, 1);
    const int most = std::min(all, kChunksMax);
    const int wanted = std::max(least, (int)std::min((long long)most, std::max(kWorkgroups / n, 1LL)));
    Cut c;
    c.tiles = (all + wanted - 1) / wanted;
    c.chunks = (all + c.tiles - 1) / c.tiles;
    // (rows times chunks of no smaller call are more)
    const size_t entries = (size_t)std::max(n * least, std::min(n * most, std::max((long long)kWorkgroups, n)));
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t x = at; at += align_up(bytes, 256); return x; };
    c.arrivals = take(n * 8 * kArrivalStep);
    c.stats = take(entries * 24);
    c.keys = take(entries * p->K * 8);
    c.total = at;
    return c;
}

template <typename T>
void launch(const LogprobArgs& a, void* stream) {
    const dim3 grid((unsigned)((long long)a.N_cap * a.chunks));
    if (a.K == 0) {
        hipLaunchKernelGGL((logprob_kernel<T, false>), grid, dim3(kThreads), 0, (hipStream_t)stream, a);
        return;
    }
    const size_t room = std::max({(size_t)a.tiles * kThreads * 4, (size_t)(a.K + kGroupsMore) * Group<T>::kN * 8, a.chunks > 1 ? (size_t)a.chunks * a.K * 8 : 0});
    hipLaunchKernelGGL((logprob_kernel<T, true>), grid, dim3(kThreads), room, (hipStream_t)stream, a);
}

int check(const fsr_logprob_params* p, const char* who) {
    if (!p) return fail(FSR_EINVAL, "%s: params is null", who);
    if (p->N_cap < 0 || p->V <= 0 || p->M < 0 || p->K < 0 || p->reserved != 0)
        return fail(FSR_EINVAL, "%s: N_cap=%d V=%d M=%d K=%d reserved=%d", who, p->N_cap, p->V, p->M, p->K, p->reserved);
    if (p->dtype != FSR_F32 && p->dtype != FSR_BF16) return fail(FSR_EUNSUP, "%s: dtype=%d", who, p->dtype);
    if (p->K > FSR_TOP_MAX) return fail(FSR_EUNSUP, "%s: K=%d alternatives (up to %d are built)", who, p->K, FSR_TOP_MAX);
    if (p->K > p->V) return fail(FSR_ESHAPE, "%s: K=%d of V=%d tokens", who, p->K, p->V);
    if (p->stride < p->V) return fail(FSR_ESHAPE, "%s: rows overlap (stride=%lld V=%d)", who, (long long)p->stride, p->V);
    if (!(p->temperature >= 1e-6) || !(p->temperature <= 1e6)) return fail(FSR_EINVAL, "%s: temperature=%g must be 1e-6 .. 1e6", who, p->temperature);
    if (p->N_cap > (1 << 22)) return fail(FSR_EUNSUP, "%s: N_cap=%d exceeds 2^22 rows", who, p->N_cap);
    if (p->V > (1 << 22)) return fail(FSR_EUNSUP, "%s: V=%d exceeds 2^22 logits", who, p->V);
    if ((long long)p->N_cap * cut(p).chunks > (1 << 23)) return fail(FSR_EUNSUP, "%s: N_cap=%d rows of V=%d logits are too many for one launch", who, p->N_cap, p->V);
    return FSR_OK;
}

}  // namespace
}  // namespace fsr

using namespace fsr;

extern "C" int fsr_logprob_workspace_bytes(const fsr_logprob_params* p, size_t* out_bytes) {
    int rc = check(p, "fsr_logprob_workspace_bytes");
    if (rc != FSR_OK) return rc;
    if (!out_bytes) return fail(FSR_EINVAL, "fsr_logprob_workspace_bytes: out_bytes is null");
    *out_bytes = cut(p).total;
    return FSR_OK;
}

extern "C" int fsr_token_logprobs(const void* logits, const int32_t* n_rows, const int32_t* tokens, float* logprobs, float* entropy, int32_t* top_ids,
                                  float* top_logprobs, const fsr_logprob_params* p, void* workspace, size_t ws_bytes, void* stream) {
    const char* who = "fsr_token_logprobs";
    int rc = check(p, who);
    if (rc != FSR_OK) return rc;
    if (p->N_cap == 0) return FSR_OK;
    if (!logits || (p->M > 0 && (!tokens || !logprobs)) || (p->K > 0 && (!top_ids || !top_logprobs)))
        return fail(FSR_EINVAL, "%s: null pointer among logits/tokens/logprobs/top_ids/top_logprobs", who);
    if ((uintptr_t)logits & (p->dtype == FSR_F32 ? 3 : 1)) return fail(FSR_EINVAL, "%s: logits must be aligned to their elements", who);
    const Cut c = cut(p);
    if (!workspace || ws_bytes < c.total) return fail(FSR_EWS, "%s: workspace %zu bytes, need %zu", who, ws_bytes, c.total);
    if ((uintptr_t)workspace & 255) return fail(FSR_EWS, "%s: workspace must be 256-byte aligned", who);
    LogprobArgs a{};
    a.logits = logits; a.n_rows = n_rows; a.tokens = tokens; a.logprobs = logprobs; a.entropy = entropy; a.top_ids = top_ids; a.top_logprobs = top_logprobs;
    a.stride = p->stride; a.N_cap = p->N_cap; a.V = p->V; a.M = p->M; a.K = p->K;
    a.scale = (float)(kLog2e / p->temperature);
    a.inv_t = 1.0 / p->temperature;
    a.chunks = c.chunks;
    a.tiles = c.tiles;
    char* w = (char*)workspace;
    a.arrivals = (unsigned long long*)(w + c.arrivals);
    a.stats = (uint64_t*)(w + c.stats);
    a.keys = (uint64_t*)(w + c.keys);
    a.call_id = c.chunks > 1 ? next_call_id() : 0;
    if (p->dtype == FSR_F32) launch<float>(a, stream);
    else launch<uint16_t>(a, stream);
    return check_launch(who);
}
