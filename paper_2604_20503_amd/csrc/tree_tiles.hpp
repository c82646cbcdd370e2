// A piece of a tree's item (row_tiles.hpp): 128 packed rows, 64 keys at a time.
//
// Tiles of the context are those of row_tiles.hpp: whole, with nothing but products in the loop.  The first tile of a piece, which finds
// the rows' references, and the tiles in which the call's own rows lie, which look at the rows' bits, take one path of their own: all
// scores, then their largest, then weights, then the second product, for 64 keys at once.  Where the values of a tile with the call's own
// rows are not all finite (each wave looks at 16 of them), the piece is given up and taken as row_tiles.hpp takes any: its keys are read twice.
// Slots of the last page that no row has yet are no part of this, whatever they hold.
#pragma once
#include "row_tiles.hpp"

namespace fsr {
namespace row_tiles {

// Where the lane's row sees a key of a tile: bit k of 64.  The words that say it are fetched a tile ahead.
struct TileWindow {
    uint32_t word[3];
    __device__ __forceinline__ void fetch(const uint32_t* row, int words, int base, int key0) {
        const int w = (key0 - base) >> 5;
#pragma unroll
        for (int k = 0; k < 3; ++k) word[k] = w + k >= 0 && w + k < words ? row[w + k] : 0u;
    }
    __device__ __forceinline__ uint64_t get(int base, int k_end, int key0) const {
        const int off = key0 - base, sh = off & 31, w = off >> 5;  // (words in front of the mask's are those of the context: all ones)
        uint32_t x[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) x[k] = w + k < 0 ? 0xffffffffu : word[k];
        const uint32_t lo = __builtin_amdgcn_alignbit(x[1], x[0], sh), hi = __builtin_amdgcn_alignbit(x[2], x[1], sh);
        const uint64_t bits = (uint64_t)hi << 32 | lo;
        const int there = k_end - key0;  // > 0
        return there >= 64 ? bits : bits & ((1ull << there) - 1);
    }
};

// Whether a wave's rows of a tile's values hold one that is not finite: 16 rows of kDv elements, in LDS.
template <class C>
__device__ __forceinline__ bool wave_odd(const char* values, int wave, int lane) {
    constexpr int kBytes = 16 * C::kDv * 2, kEach = kBytes / (kWave * 16);
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(values + wave * kBytes + (i * kWave + lane) * 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) odd |= (x[k] & 0x7f807f80u) + 0x00800080u;  // (an exponent of all ones carries)
    }
    return __any((odd & 0x80008000u) != 0);
}

// 64 keys of any tile whose values are finite; window: the keys that the lane's row sees.
template <class C>
__device__ __forceinline__ void take_tree_tile(Rows<C>& w, const char* buf, uint64_t window, float scale_log2, int lane) {
    typedef Rows<C> R;
    constexpr int kSteps = R::kHeadSteps;
    static_assert(R::kTailSteps == 0, "trees have keys of one part");
    f32x16 z[2] = {zeros(), zeros()};
    in_turn<2 * kSteps, 8, bf16x8>(
        [&](int k) __attribute__((always_inline)) {
            const int s = k >> 1;
            return *reinterpret_cast<const bf16x8*>(buf + C::kHeadAt + (k & 1) * 32 * C::kHead * 2 + w.k_at[s % R::kOwnK] + (s / R::kOwnK) * 256);
        },
        [&](int k, bf16x8 x) __attribute__((always_inline)) { z[k & 1] = product(x, w.q[k >> 1], z[k & 1]); }, [](int) {});
    if (!__all(window == ~0ull)) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int bits = (int)((uint32_t)(window >> (32 * b)) >> (4 * (lane >> 5)));
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t sees = (uint32_t)__builtin_amdgcn_sbfe(bits, 8 * (e >> 2) + (e & 3), 1);  // all ones or none
                const float x = z[b][e];  // (a bit cast of the element itself takes element 0)
                z[b][e] = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, x) & sees) | (0xff800000u & ~sees));
            }
        }
    }
    const float top = fmaxf(largest(z[0]), largest(z[1]));
    const bool ahead = exponent(top, w.of, scale_log2) > 0.0f;
    if (__any(ahead)) {
        const Reference old = w.of;
        if (ahead) w.of = reference_for(top, scale_log2);
        const float alpha = !ahead || old.log2 == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(distance(old, w.of, scale_log2));
        w.l *= alpha;
#pragma unroll
        for (int b = 0; b < R::kBlocks; ++b) w.acc[b] *= alpha;
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) w.l += weights_of(z[b], w.of, scale_log2);
    bf16x8 hi[4], lo[C::kPair ? 4 : 1];
#pragma unroll
    for (int s = 0; s < 4; ++s) hi[s] = operand_of(z[s >> 1], s & 1);
    if constexpr (C::kPair) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) z[b][e] -= (float)(__bf16)z[b][e];
#pragma unroll
        for (int s = 0; s < 4; ++s) lo[s] = operand_of(z[s >> 1], s & 1);
    }
    in_turn<4 * R::kBlocks, 6, s16x8>([&](int k) __attribute__((always_inline)) { return values_of<C>(w, buf, k / R::kBlocks >> 1, k / R::kBlocks & 1, k % R::kBlocks); },
                                      [&](int k, s16x8 v) __attribute__((always_inline)) {
                                          const int b = k % R::kBlocks, s = k / R::kBlocks;
                                          w.acc[b] = product(__builtin_bit_cast(bf16x8, v), hi[s], w.acc[b]);
                                          if constexpr (C::kPair) w.acc[b] = product(__builtin_bit_cast(bf16x8, v), lo[s], w.acc[b]);
                                      },
                                      [](int) {});
}

// False: the piece is to be taken by run_tiled, without its fast loop (as there; or a value that some row does not see is not finite).
template <class C>
__device__ __forceinline__ bool run_tree(const Args& a, const Piece& p, char* buf0, char* buf1, int* flags) {
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), li = lane & 31, h = lane >> 5;
    const int n_packed = p.q.rows * a.G, first = p.rt * C::kM + wave * 32;
    const bool active = first < n_packed;  // a wave without rows helps to load
    typedef Rows<C> R;
    R w;
    w.of = Reference{0.0f, -INFINITY};
    w.l = 0.0f;
    w.seen = p.q.k_end - 1;
    w.place_operands(lane);
#pragma unroll
    for (int b = 0; b < R::kBlocks; ++b) w.acc[b] = zeros();
    TileLoads<C> loads;
    loads.place_lane(a, lane);
    int t = p.t0;
    auto load_all = [&](char* to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < TileLoads<C>::kEach; ++i) loads.issue(i, a, p, to, wave, lane);
    };
    __syncthreads();  // nobody reads the buffers any more
    if (t < p.t1) loads.find(a, p, t, wave, lane);
    w.tree = a.tree;
    if (active) {
        const Place at = place_of(a, p.q.row0, p.hk, min(first + li, n_packed - 1));
        const uint16_t* qp = (const uint16_t*)a.q + ((size_t)at.row * a.H + at.head) * C::kDk;
#pragma unroll
        for (int s = 0; s < C::kDk / 16; ++s) w.q[s] = *reinterpret_cast<const bf16x8*>(qp + 16 * s + 8 * h);
        w.tree = a.tree + (size_t)at.row * a.tree_words;
    }
    if (t < p.t1) {
        loads.take(a, p);
        load_all(buf0);
        loads.find(a, p, min(t + 1, p.t1 - 1), wave, lane);
        const int whole_until = min(p.t1, p.q.base / C::kKeys);  // tiles of the context alone
        TileWindow windows;
        windows.fetch(w.tree, a.tree_words, p.q.base, max(t, whole_until) * C::kKeys);
        // A tile of the fast loop; false: a reference moves, and the tile is still to be added (the next one's loads are under way).
        auto step = [&](const char* now, char* then) __attribute__((always_inline)) {
            arrive();  // (and nobody reads the other buffer any more)
            loads.take(a, p);
            loads.find(a, p, min(t + 2, p.t1 - 1), wave, lane);  // (behind the last tile this one is loaded again: a load too many costs less than asking)
            static_assert(TileLoads<C>::kEach <= 2 * (R::kHeadSteps + R::kTailSteps), "a load beside a product");
            const bool ahead = take_tile<C>(w, now, a.scale_log2, [&](int i) __attribute__((always_inline)) {
                if (i < TileLoads<C>::kEach) loads.issue(i, a, p, then, wave, lane);
            });
            t += !ahead;
            return !ahead;
        };
        bool loaded = false;  // the next tile's loads have been issued
        while (t < p.t1) {
            const bool odd = (t - p.t0) & 1;
            const char* now = odd ? buf1 : buf0;
            if (!loaded) {
                arrive();
                loads.take(a, p);
                loads.find(a, p, min(t + 2, p.t1 - 1), wave, lane);
                load_all(odd ? buf0 : buf1);
            }
            loaded = false;
            uint64_t window = ~0ull;
            if (t >= whole_until) {  // (for the whole workgroup: a value must not meet the weight 0 of a row that does not see it)
                window = windows.get(p.q.base, p.q.k_end, t * C::kKeys);
                windows.fetch(w.tree, a.tree_words, p.q.base, (t + 1) * C::kKeys);
                const bool mine = wave_odd<C>(now + C::kVAt, wave, lane);
                if (lane == 0) flags[wave] = mine;
                lds_barrier();
                if (uniform(flags[0] | flags[1] | flags[2] | flags[3])) {
                    __builtin_amdgcn_s_waitcnt(0x0f70);
                    return false;
                }
            }
            if (active) take_tree_tile<C>(w, now, window, a.scale_log2, lane);
            ++t;
            // all the others: here the sums are the products' alone (where something else may touch them, the compiler makes a second
            // set and copies them in every tile)
            const bool near = uniform((int)__any(w.of.raw != 0.0f)) == 0;
            if (!odd && near && active) {
                w.of.raw = 0.0f;  // (known, and in no register of the loop)
                while (t < whole_until) {
                    if (!step(buf1, buf0)) { loaded = true; break; }
                    if (t >= whole_until) break;
                    if (!step(buf0, buf1)) { loaded = true; break; }
                }
            }
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);  // the load too many has its place until it has come
    }
    if constexpr (C::kPair) {  // (of one tile of the context too: its values have not been looked at)
        float odd = 0.0f;
#pragma unroll
        for (int b = 0; b < R::kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) odd = fmaf(w.acc[b][e], 0.0f, odd);
        const int mine = __any(odd != 0.0f);
        __syncthreads();
        if (lane == 0) flags[wave] = mine;
        __syncthreads();
        if (uniform(flags[0] | flags[1] | flags[2] | flags[3])) return false;
    }
    w.l += other_half(w.l);
    if (active && first + li < n_packed)
        hand_over<C>(a, p, wave * 32 + li, h == 0, w.of, w.l, [&](auto put) {
#pragma unroll
            for (int b = 0; b < R::kBlocks; ++b)
#pragma unroll
                for (int g = 0; g < 4; ++g) put(32 * b + 8 * g + 4 * h, f32x4{w.acc[b][4 * g], w.acc[b][4 * g + 1], w.acc[b][4 * g + 2], w.acc[b][4 * g + 3]});
        });
    return true;
}

// Joins the pieces of an item.  Sums lie as the lanes of a wave held them, and so they are read: a lane has one row, whose statistics of all
// pieces it takes for itself, and four columns of it at a time.  A workgroup joins the rows of one wave, each of its waves a quarter of the
// columns.  (With a row's columns in a row, stores were of 32 bytes a row, 4500 cycles a piece, and a wave's lanes had to exchange
// statistics.)  Eight pieces are under way at once (four: 12 rows behind 777 tokens, 32/8 heads, 18.5 us, not 16.4); with sixteen, or the
// columns over more workgroups, which compute the same weights again, 16 requests of 24-64 rows took up to 14 us more, of 82.
template <class C>
__global__ __launch_bounds__(kThreads) void join_tree_kernel(Args a) {
    constexpr int kGroups = C::kDv / C::kPartColumns, kMine = kGroups / kWaves, kChunk = 8;
    static_assert(kGroups % kWaves == 0, "a share of the columns for each wave");
    constexpr Reference kNone{-INFINITY, 0.0f};
    const int32_t* desc = a.desc + (size_t)blockIdx.x * kDescInts;
    const int pieces = desc[0], row0 = desc[1], hk = desc[2], rt = desc[3], rows = desc[4], first_slot = desc[5], second_slot = desc[6], step = desc[7];
    if (pieces <= 0 || (int)blockIdx.y * C::kPartRows >= rows) return;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), r = blockIdx.y * C::kPartRows + lane % C::kPartRows;
    auto slot = [&](int k) { return k == 0 ? first_slot : second_slot + (k - 1) * step; };
    auto sums_of = [&](int k) { return reinterpret_cast<const f32x4*>(a.part_o + (size_t)slot(k) * a.m_cap * C::kDv) + (blockIdx.y * kGroups + wave * kMine) * 64 + lane; };
    f32x4 o[kMine];
#pragma unroll
    for (int c = 0; c < kMine; ++c) o[c] = f32x4{0, 0, 0, 0};
    float l = 0.0f;
    Reference of = kNone;
    for (int first = 0; first < pieces; first += kChunk) {
        const int n = min(pieces - first, kChunk);
        f32x4 stats[kChunk], y[kChunk][kMine];
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
            if (i < n) stats[i] = reinterpret_cast<const f32x4*>(a.part_ml)[(size_t)slot(first + i) * a.m_cap + min(r, rows - 1)];
        auto fetch = [&]() __attribute__((always_inline)) {  // (in two plain loops, of which the compiler makes one: 8 requests in fp32 17.6 us, not 15.1)
#pragma unroll
            for (int i = 0; i < kChunk; ++i)
                if (i < n) {
                    const f32x4* x = sums_of(first + i);
#pragma unroll
                    for (int c = 0; c < kMine; ++c) y[i][c] = x[c * 64];
                }
        };
        fetch();
        // Any number near the furthest reference will do; where powers of two are too coarse for one, it is that reference itself.
        float top = fmaf(of.raw, a.scale_log2, of.log2);
        Reference furthest = of;
#pragma unroll
        for (int i = 0; i < kChunk; ++i) {
            if (i >= n) break;
            if (stats[i][2] == 0.0f) continue;  // (a piece without a visible key)
            const Reference pm{stats[i][0], stats[i][1]};
            top = fmaxf(top, fmaf(pm.raw, a.scale_log2, pm.log2));
            if (distance(pm, furthest, a.scale_log2) > 0.0f) furthest = pm;
        }
        const Reference use = fabsf(top) <= kNear ? Reference{0.0f, top} : furthest;
        const float before = l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(distance(of, use, a.scale_log2));
        l *= before;
#pragma unroll
        for (int c = 0; c < kMine; ++c) o[c] *= before;
        float w[kChunk];
#pragma unroll
        for (int i = 0; i < kChunk; ++i) {
            if (i >= n) break;
            const float pl = stats[i][2];
            w[i] = pl == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(distance(Reference{stats[i][0], stats[i][1]}, use, a.scale_log2));
            l = fmaf(w[i], pl, l);
        }
        of = l == 0.0f ? kNone : use;
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
            if (i < n)
#pragma unroll
                for (int c = 0; c < kMine; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[c][e] = fmaf(w[i], y[i][c][e], o[c][e]);
    }
    if (r >= rows) return;
    const float inv = inverse(l);
    const Place to = place_of(a, row0, hk, rt * C::kM + r);
    const size_t row = (size_t)to.row * a.H + to.head;
    // (Tiled: group b, g of a lane's half h are columns 32 b + 8 g + 4 h; Simple: of lane group lg 16 b + 4 lg)
    typename C::Out* out = (typename C::Out*)a.out + row * C::kDv + wave * kMine * C::kPartColumns + (lane / C::kPartRows) * 4;
#pragma unroll
    for (int c = 0; c < kMine; ++c) store4(out + c * C::kPartColumns, o[c] * inv);
    if (a.lse && wave == 0 && lane < C::kPartRows) a.lse[row] = log_sum<C::kOp>(of, l, a.scale);
}

template <class C>
void launch_tree_join(const Args& a, hipStream_t s) {
    const int rows = std::min(a.m_cap, C::kM);
    hipLaunchKernelGGL((join_tree_kernel<C>), dim3(a.nb, (rows + C::kPartRows - 1) / C::kPartRows), dim3(kThreads), 0, s, a);
}

template <int KH, int KT, int DV, class OUT, bool PAGES16>
struct Pieces<Tiled<kTree, KH, KT, DV, OUT, PAGES16>> {
    typedef Tiled<kTree, KH, KT, DV, OUT, PAGES16> C;
    static constexpr int kShared = C::kWaves * sizeof(int);
    static __device__ __forceinline__ bool take(const Args& a, const Piece& p, char* buf0, char* buf1, int* more, bool fast) {
        return fast ? run_tree<C>(a, p, buf0, buf1, more) : run_tiled<C>(a, p, buf0, buf1, false);
    }
};

}  // namespace row_tiles
}  // namespace fsr
