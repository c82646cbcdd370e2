// bf16 attention on a latent cache: keys of 512 + 64 elements whose first 512 are the values, all query heads on one stream.
//
// 32 rows of such sums and queries fill a wave's registers (256 + 144 of 512 a lane), with nothing left to feed the matrix cores from.
// So a workgroup takes 64 rows in four waves, two for each 32 rows: of 64 keys each takes the scores of 32, hands its weights to the
// other through LDS, and then multiplies all 64 keys' weights with its half of the values' columns (128 + 144 registers).  What
// LDS has to deliver per tile, keys once per two waves and values once per two waves, is 370 KB against 2176 cycles of the matrix
// cores (2900 cycles at 128 bytes each); with 16 rows a wave it would be 626 KB.
//
// The exponent reference of a row has to be common to both waves.  It is kept kAhead powers of two above the largest score seen and
// changed only in a tile where a score overtakes it, the first one for the most part, with two more barriers.
#pragma once
#include "row_tiles.hpp"

namespace fsr {
namespace row_tiles {

template <int KH, int KT, class OUT>
struct Latent {
    static constexpr int kOp = kLatent, kHead = KH, kTail = KT, kDk = KH + KT, kDv = KH;
    static constexpr bool kPair = sizeof(OUT) == 4;
    static constexpr int kM = 64, kKeys = 64, kBlockThreads = 256, kWaves = 4, kPerUnit = 1;
    static constexpr int kHeadAt = 0, kTailAt = kKeys * KH * 2, kBuf = kTailAt + kKeys * KT * 2;
    typedef uint16_t In;
    typedef OUT Out;
};

struct LatentShared {     // what the waves of a workgroup tell each other
    uint16_t p[64][64];   // weights [row][key], 16-byte chunks of a row permuted
    float top[4][32];     // largest score of a row among a wave's keys; at the end its sum of weights
    int flags[4];         // by wave: 1: a score is ahead of its reference, 2: scores that are not finite among masked ones
};

template <class C>
struct LatentRows {
    static constexpr int kHeadSteps = C::kHead / 16, kTailSteps = C::kTail / 16, kBlocks = C::kDv / 64;  // (half the columns)
    bf16x8 q[kHeadSteps + kTailSteps];
    f32x16 acc[kBlocks];
    float m, l;
    int seen;
    int k_at[8], tail_at[kTailSteps], v_at[4], p_write[4], p_read[4];

    __device__ __forceinline__ void place_operands(int lane, int rows, int part) {
        const int li = lane & 31, h = lane >> 5;
        constexpr int CH = C::kHead / 8, CT = C::kTail / 8;
#pragma unroll
        for (int s = 0; s < 8; ++s) k_at[s] = (32 * part + li) * CH * 16 + (((2 * s + h) ^ permutation<CH>(li)) << 4);
#pragma unroll
        for (int s = 0; s < kTailSteps; ++s) tail_at[s] = (32 * part + li) * CT * 16 + (((2 * s + h) ^ permutation<CT>(li)) << 4);
        const int g = lane & 15, r = 8 * h + (g >> 2), column = lane & 16;
#pragma unroll
        for (int b = 0; b < 4; ++b)
            v_at[b] = part * C::kHead + r * CH * 16 + (g & 1) * 8 + ((((32 * b + column) / 8 + ((g & 3) >> 1)) ^ permutation<CH>(r)) << 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            p_write[k] = (32 * rows + li) * 128 + (((4 * part + k) ^ (li & 7)) << 4) + 8 * h;  // keys 8 k + 4 h .. of the wave's
            p_read[k] = (32 * rows + li) * 128 + (((2 * k + h) ^ (li & 7)) << 4);              // keys 16 k + 8 h .. of all
        }
    }
};

template <class C>
__device__ __forceinline__ void write_weights(const LatentRows<C>& w, char* p, const float (&z)[16]) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
        *reinterpret_cast<u32x2*>(p + w.p_write[k]) = u32x2{bf16_bits(z[4 * k]) | (bf16_bits(z[4 * k + 1]) << 16), bf16_bits(z[4 * k + 2]) | (bf16_bits(z[4 * k + 3]) << 16)};
}

// acc += V^T P^T for the wave's half of the columns.
template <class C>
__device__ __forceinline__ void second_product(LatentRows<C>& w, const char* buf, const char* p, bool careful) {
    typedef LatentRows<C> R;
    constexpr int kRow = C::kHead * 2;
    bf16x8 weights[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) weights[s] = *reinterpret_cast<const bf16x8*>(p + w.p_read[s]);
    // (keys 4 .. 7 of eight: the permutation of their rows differs in the bit that tells apart blocks b and b ^ 2)
    auto values = [&](int s, int b) __attribute__((always_inline)) {
        const char* at = buf + C::kHeadAt + 16 * s * kRow + (b / 4) * 256;
        return transposed(at + w.v_at[b % 4], at + 4 * kRow + w.v_at[(b % 4) ^ 2]);
    };
    if (!careful) {
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int b = 0; b < R::kBlocks; ++b) w.acc[b] = product(__builtin_bit_cast(bf16x8, values(s, b)), weights[s], w.acc[b]);
        return;
    }
    // values that are not finite among masked ones: see take_keys
#pragma unroll
    for (int b = 0; b < R::kBlocks; ++b) {
#pragma unroll
        for (int s = 0; s < 4; ++s) w.acc[b] = product(elements(values(s, b), kFinite), weights[s], w.acc[b]);
#pragma unroll 1
        for (int kind = kUp; kind <= kNan; ++kind) {
            f32x16 t = zeros();
#pragma unroll
            for (int s = 0; s < 4; ++s) t = product(elements(values(s, b), kind), weights[s], t);
            put_odd(w.acc[b], t, kind);
        }
    }
}

// One tile of 64 keys from `key0` on.  All waves pass the same barriers; those of rows that see none of the keys (not `live`) do no more.
template <class C>
__device__ __forceinline__ void take_tile(LatentRows<C>& w, const char* buf, LatentShared& sh, int key0, bool live, bool masked, float scale_log2, int lane,
                                          int wave) {
    typedef LatentRows<C> R;
    const int li = lane & 31, h = lane >> 5, part = wave & 1;
    char* p = reinterpret_cast<char*>(sh.p);
    float z[16], x[16], sum = 0.0f, top = -INFINITY;
    auto weigh = [&]() __attribute__((always_inline)) {
        const float m = w.m == -INFINITY ? 0.0f : w.m;
        sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            x[e] = __builtin_amdgcn_exp2f(fmaf(z[e], scale_log2, -m));
            sum += x[e];
        }
        write_weights<C>(w, p, x);
    };
    int flags = 0;
    if (live) {
        f32x16 scores = zeros();
#pragma unroll
        for (int s = 0; s < R::kHeadSteps; ++s)
            scores = product(*reinterpret_cast<const bf16x8*>(buf + C::kHeadAt + w.k_at[s % 8] + (s / 8) * 256), w.q[s], scores);
#pragma unroll
        for (int s = 0; s < R::kTailSteps; ++s)
            scores = product(*reinterpret_cast<const bf16x8*>(buf + C::kTailAt + w.tail_at[s]), w.q[R::kHeadSteps + s], scores);
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = scores[e];
        if (masked) {
            float odd = 0.0f;  // a value that is not finite is in its key, too, and has made the key's scores infinite or NaN
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                odd += z[e] - z[e];
                z[e] = key0 + 32 * part + 8 * (e >> 2) + 4 * h + (e & 3) <= w.seen ? z[e] : -INFINITY;
            }
            if (__any(odd != 0.0f)) flags = 2;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, z[e]);
        top = fmaxf(top, other_half(top)) * scale_log2;
        if (__any(top > w.m)) flags |= 1;
        weigh();
    }
    if (lane == 0) sh.flags[wave] = flags;
    __syncthreads();
    const int rows01 = uniform(sh.flags[0] | sh.flags[1]), rows23 = uniform(sh.flags[2] | sh.flags[3]);
    if ((rows01 | rows23) & 1) {  // some row's reference moves
        if (h == 0) sh.top[wave][li] = top;
        __syncthreads();
        if (live) {
            const float both = fmaxf(sh.top[wave & 2][li], sh.top[wave | 1][li]), old = w.m;
            if (both > old) w.m = both + kAhead;
            const float alpha = w.m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(old - w.m);
            w.l *= alpha;
#pragma unroll
            for (int b = 0; b < R::kBlocks; ++b) w.acc[b] *= alpha;
            weigh();
        }
        __syncthreads();
    }
    w.l += sum;
    const bool careful = ((wave & 2 ? rows23 : rows01) & 2) != 0;
    if (live) second_product<C>(w, buf, p, careful);
    if constexpr (C::kPair) {
        __syncthreads();
        if (live) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] -= (float)(__bf16)x[e];
            write_weights<C>(w, p, x);
        }
        __syncthreads();
        // (a weight's rest has no infinite values to meet that its leading part has not met: they are left out)
        if (live) second_product<C>(w, buf, p, careful);
    }
}

template <class C>
__device__ __forceinline__ void run_latent(const Args& a, const Piece& p, char* buf0, char* buf1, LatentShared& sh) {
    typedef LatentRows<C> R;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), li = lane & 31, h = lane >> 5, part = wave & 1;
    const int n_packed = p.q.rows * a.G, first = p.rt * C::kM + (wave >> 1) * 32;
    const bool active = first < n_packed;  // a wave without rows helps to load
    R w;
    w.m = -INFINITY;
    w.l = 0.0f;
    w.seen = -1;
    w.place_operands(lane, wave >> 1, part);
    auto find = [&](int t) { return find_key<C::kOp>(a, p.q, min(p.q.k_begin + t * C::kKeys + lane, p.q.k_end - 1)); };
    __syncthreads();  // nobody reads the buffers any more
    int t = p.t0;
    Where next{};
    if (t < p.t1) {
        load_tile<C>(a, p, slot_of<C::kOp>(a, find(t)), buf0, wave, lane);
        next = find(min(t + 1, p.t1 - 1));
    }
    int seen_first = 0, seen_last = -1;  // by the wave's first and last row
    if (active) {
        const int r = min(first + li, n_packed - 1);
        const Place at = place_of(a, p.q.row0, p.hk, r);
        const uint16_t* qp = (const uint16_t*)a.q + ((size_t)at.row * a.H + at.head) * C::kDk;
#pragma unroll
        for (int s = 0; s < C::kDk / 16; ++s) w.q[s] = *reinterpret_cast<const bf16x8*>(qp + 16 * s + 8 * h);
        w.seen = last_key(a, p.q, r);
        seen_first = last_key(a, p.q, first);
        seen_last = last_key(a, p.q, min(first + 31, n_packed - 1));
    }
#pragma unroll
    for (int b = 0; b < R::kBlocks; ++b) w.acc[b] = zeros();
    auto step = [&](char* now, char* then) __attribute__((always_inline)) {
        arrive();  // (and nobody reads the other buffer any more)
        if (t + 1 < p.t1) {
            load_tile<C>(a, p, slot_of<C::kOp>(a, next), then, wave, lane);
            next = find(min(t + 2, p.t1 - 1));
        }
        const int key0 = p.q.k_begin + t * C::kKeys;
        take_tile<C>(w, now, sh, key0, key0 <= seen_last, key0 + C::kKeys - 1 > seen_first, a.scale_log2, lane, wave);
        return ++t < p.t1;
    };
    if (t < p.t1)
        while (step(buf0, buf1) && step(buf1, buf0)) {}
    w.l += other_half(w.l);
    __syncthreads();
    if (h == 0) sh.top[wave][li] = w.l;
    __syncthreads();
    if (active && first + li < n_packed)
        hand_over<C>(a, p, (wave >> 1) * 32 + li, h == 0 && part == 0, w.m * kLn2, sh.top[wave & 2][li] + sh.top[wave | 1][li], [&](auto put) {
#pragma unroll
            for (int b = 0; b < R::kBlocks; ++b)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    put(part * (C::kDv / 2) + 32 * b + 8 * g + 4 * h, f32x4{w.acc[b][4 * g], w.acc[b][4 * g + 1], w.acc[b][4 * g + 2], w.acc[b][4 * g + 3]});
        });
}

template <class C>
__global__ __launch_bounds__(C::kBlockThreads, 1) void latent_kernel(Args a) {
    __shared__ __align__(1024) char buf0[C::kBuf];
    __shared__ __align__(1024) char buf1[C::kBuf];
    __shared__ __align__(1024) LatentShared sh;
    const int share = share_of_block(blockIdx.x, a.nb);
    const Line line = find_share<C>(a, share, reinterpret_cast<long long*>(buf0));
    walk<C>(a, share, line, [&](const Piece& p) { run_latent<C>(a, p, buf0, buf1, sh); });
}
template <int KH, int KT, class OUT>
struct Kernel<Latent<KH, KT, OUT>> {
    static constexpr auto run = latent_kernel<Latent<KH, KT, OUT>>;
};

}  // namespace row_tiles
}  // namespace fsr
