// Workgroups on the CPU, for tests of how a kernel's waves hand each other data: every lane is a fiber, operations of a wave wait for
// its 64 lanes, barriers for the whole workgroup, and in between waves run as far as they get, one before the other in an order that
// the test chooses.  What a kernel leaves to chance, by a barrier that is missing, then goes wrong every time.  Workgroups run one after
// the other; of HIP there is what the kernels under test use.
#pragma once
#include <ucontext.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <memory>
#include <random>
#include <vector>

#define __device__
#define __global__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __align__(n) __attribute__((aligned(n)))
#define __HIP_MEMORY_SCOPE_AGENT 0

typedef void* hipStream_t;
typedef int hipError_t;
constexpr hipError_t hipSuccess = 0;
inline hipError_t hipGetLastError() { return hipSuccess; }
inline const char* hipGetErrorString(hipError_t) { return ""; }
struct dim3 {
    unsigned x, y, z;
    dim3(unsigned x = 1, unsigned y = 1, unsigned z = 1) : x(x), y(y), z(z) {}
};

namespace workgroup {

constexpr int kLanes = 64;

struct Lane {
    ucontext_t context;
    int id, waits_for_wave = -1, waits_for_all = -1;  // rounds of the wave's operations, of the workgroup's barriers
    bool done = false;
};
struct Wave {
    int round = 0, arrived = 0;
    uint64_t posted[2][kLanes];  // (a lane is one round ahead of another at most)
};
struct State {
    dim3 block, block_idx;
    std::vector<Lane> lanes;
    std::vector<Wave> waves;
    int round = 0, arrived = 0;
    Lane* now = nullptr;
    ucontext_t scheduler;
    const std::function<void()>* body = nullptr;
};
inline State state;
inline int order = 0;  // of waves: 0 ascending, 1 descending, else shuffled by this seed
alignas(1024) inline char dynamic_lds[65536];
constexpr size_t kStack = 128 << 10;
inline std::unique_ptr<char[]> stacks;
inline size_t stacks_of = 0;

inline void yield() { swapcontext(&state.now->context, &state.scheduler); }
inline void run_lane() {
    (*state.body)();
    state.now->done = true;
    yield();
}

inline void barrier() {
    Lane& me = *state.now;
    if (++state.arrived == (int)state.lanes.size()) {
        state.arrived = 0;
        ++state.round;
    } else {
        me.waits_for_all = state.round;
        yield();
    }
}

// Posts a value of every lane; behind it all of the wave's are there.
inline const uint64_t* exchange(uint64_t mine) {
    Lane& me = *state.now;
    Wave& w = state.waves[me.id / kLanes];
    const int round = w.round;
    w.posted[round & 1][me.id % kLanes] = mine;
    if (++w.arrived == kLanes) {
        w.arrived = 0;
        ++w.round;
    } else {
        me.waits_for_wave = round;
        yield();
    }
    return w.posted[round & 1];
}

inline bool can_run(const Lane& l) {
    return !l.done && l.waits_for_all != state.round && l.waits_for_wave != state.waves[l.id / kLanes].round;
}

inline void launch(dim3 grid, dim3 block, size_t lds, const std::function<void()>& body) {
    if (block.x % kLanes != 0 || lds > sizeof dynamic_lds) abort();
    const int waves = block.x / kLanes;
    if (stacks_of < block.x) stacks.reset(new char[block.x * kStack]), stacks_of = block.x;
    std::vector<int> turn(waves);
    std::mt19937 random(order);
    for (unsigned b = 0; b < grid.x; ++b) {
        state = State{};
        state.block = block;
        state.block_idx = dim3(b, 0, 0);
        state.body = &body;
        state.lanes.resize(block.x);
        state.waves.resize(waves);
        memset(dynamic_lds, 0xa5, sizeof dynamic_lds);
        for (int w = 0; w < waves; ++w) turn[w] = order == 1 ? waves - 1 - w : w;
        if (order > 1) std::shuffle(turn.begin(), turn.end(), random);
        for (unsigned t = 0; t < block.x; ++t) {
            Lane& l = state.lanes[t];
            l.id = t;
            getcontext(&l.context);
            l.context.uc_stack.ss_sp = stacks.get() + t * kStack;
            l.context.uc_stack.ss_size = kStack;
            l.context.uc_link = &state.scheduler;
            makecontext(&l.context, run_lane, 0);
        }
        for (bool ran = true; ran;) {  // the first wave that can run does, until all of its lanes wait
            ran = false;
            for (int w = 0; w < waves && !ran; ++w)
                for (int k = 0; k < kLanes; ++k) {
                    Lane& l = state.lanes[turn[w] * kLanes + k];
                    if (!can_run(l)) continue;
                    l.waits_for_all = l.waits_for_wave = -1;
                    state.now = &l;
                    swapcontext(&state.scheduler, &l.context);
                    ran = true;
                }
        }
        for (const Lane& l : state.lanes)
            if (!l.done) {
                fprintf(stderr, "workgroup %u: lane %d waits for ever\n", b, l.id);
                abort();
            }
    }
}

template <class T>
inline uint64_t bits(T x) {
    uint64_t b = 0;
    memcpy(&b, &x, sizeof x);
    return b;
}
template <class T>
inline T as(uint64_t b) {
    T x;
    memcpy(&x, &b, sizeof x);
    return x;
}
inline int lane() { return state.now->id % kLanes; }
inline unsigned long long ballot(bool x) {
    const uint64_t* all = exchange(x);
    unsigned long long b = 0;
    for (int k = 0; k < kLanes; ++k) b |= (unsigned long long)all[k] << k;
    return b;
}
// Moves between the lanes of a row of 16 and between rows, as the codes of DPP have them.
inline int move(int old, int x, int code, int rows, int, bool zero) {
    const uint64_t* all = exchange((uint32_t)x);
    const int at = lane(), row = at / 16;
    if (!(rows >> row & 1)) return old;
    int from = -1;
    if (code < 0x100) from = (at & ~3) + (code >> 2 * (at & 3) & 3);
    else if (code > 0x110 && code < 0x120) from = at % 16 >= code - 0x110 ? at - (code - 0x110) : -1;
    else if (code == 0x142) from = row > 0 ? 16 * row - 1 : -1;
    else if (code == 0x143) from = row > 1 ? 31 : -1;
    else abort();
    return from >= 0 ? (int)(uint32_t)all[from] : zero ? 0 : old;
}

struct Index {
    uint32_t x, y, z;
};

}  // namespace workgroup

#define threadIdx (::workgroup::Index{(uint32_t)::workgroup::state.now->id, 0, 0})
#define blockIdx (::workgroup::state.block_idx)
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) \
    ((void)(stream), ::workgroup::launch(grid, block, lds, [=] { kernel(__VA_ARGS__); }))

inline void __syncthreads() { ::workgroup::barrier(); }
inline unsigned long long __ballot(int x) { return ::workgroup::ballot(x != 0); }
inline int __any(int x) { return ::workgroup::ballot(x != 0) != 0; }
inline int __all(int x) { return ::workgroup::ballot(x != 0) == ~0ull; }
template <class T>
inline T __shfl(T x, int from, int) { return ::workgroup::as<T>(::workgroup::exchange(::workgroup::bits(x))[from & 63]); }
template <class T>
inline T __shfl_xor(T x, int o, int) { return __shfl(x, ::workgroup::lane() ^ o, 64); }
template <class T>
inline T __shfl_up(T x, int o, int) { return __shfl(x, ::workgroup::lane() >= o ? ::workgroup::lane() - o : ::workgroup::lane(), 64); }
inline int __popc(unsigned x) { return __builtin_popcount(x); }
inline int __popcll(unsigned long long x) { return __builtin_popcountll(x); }
inline int __clzll(long long x) { return x ? __builtin_clzll((unsigned long long)x) : 64; }
inline int __ffsll(unsigned long long x) { return __builtin_ffsll((long long)x); }
template <class T>
inline T min(T x, T y) { return y < x ? y : x; }
template <class T>
inline T max(T x, T y) { return x < y ? y : x; }
template <class T>
inline T atomicAdd(T* p, T x) { const T old = *p; *p += x; return old; }
template <class T>
inline T atomicMin(T* p, T x) { const T old = *p; if (x < old) *p = x; return old; }
template <class T>
inline T atomicCAS(T* p, T expected, T x) { const T old = *p; if (old == expected) *p = x; return old; }

#define __hip_atomic_store(p, x, order, scope) ((void)(*(p) = (x)))
#define __hip_atomic_load(p, order, scope) (*(p))
#define __builtin_amdgcn_update_dpp(old, x, code, rows, banks, zero) ::workgroup::move(old, x, code, rows, banks, zero)
#define __builtin_amdgcn_readlane(x, from) ((int)(uint32_t)::workgroup::exchange((uint32_t)(x))[from])
#define __builtin_amdgcn_readfirstlane(x) __builtin_amdgcn_readlane(x, 0)
#define __builtin_amdgcn_exp2f(x) exp2f(x)
#define __builtin_amdgcn_logf(x) log2f(x)
#define __builtin_canonicalizef(x) ((x) != (x) ? NAN : (x))
#define __builtin_amdgcn_cvt_pk_fp8_f32(x, y, old, high) (abort(), 0)  // (no test needs it)
inline int __builtin_frexp_exp(float x) { int e; return frexpf(x, &e), e; }
inline float __builtin_frexp_mant(float x) { int e; return frexpf(x, &e); }
#define __builtin_amdgcn_frexp_expf(x) __builtin_frexp_exp(x)
#define __builtin_amdgcn_frexp_mantf(x) __builtin_frexp_mant(x)
