// bf16 attention on a latent cache: keys of 512 + 64 elements whose first 512 are the values, all query heads on one stream.
//
// 32 rows of such sums and queries fill a wave's registers (256 + 144 of 512 a lane), with nothing left to feed the matrix cores from.
// So a workgroup takes 64 rows in four waves, two for each 32 rows: of 64 keys each takes the scores of 32, hands its weights to the
// other through LDS, and then multiplies all 64 keys' weights with its half of the values' columns (128 + 144 registers).  What
// LDS has to deliver per tile, keys once per two waves and values once per two waves, is 370 KB against 2176 cycles of the matrix
// cores (2900 cycles at 128 bytes each); with 16 rows a wave it would be 626 KB.
//
// Measured: 4350 cycles a tile whose keys come from the cache, scores 1660, weights 690, second product 1500 and three barriers one after the
// other: with one wave a SIMD nothing runs beside them, and that, not LDS, is the bound.  64 requests of 512-4096 keys, 1-4 rows, 128 heads:
// 210-219 us by card, 529-507 TFLOP/s; 32 of 1024-8192 keys, 16 heads: 75-82 us, 2.2-2.0 TB/s.  The kernels of 512 elements use all 512
// registers, and what is set up once a piece (addresses, schedule) and the general tiles spill 110-200 more; the loop over whole tiles does not.
//
// The exponent reference of a row has to be common to both waves.  It is kept kAhead powers of two above the largest score seen and
// changed only in a tile where a score overtakes it, the first one for the most part, with two more barriers.
#pragma once
#include "row_tiles.hpp"

namespace fsr {
namespace row_tiles {

// PAGES16: pages hold a multiple of 16 tokens.
template <int KH, int KT, class OUT, bool PAGES16>
struct Latent {
    static constexpr int kOp = kLatent, kHead = KH, kTail = KT, kDk = KH + KT, kDv = KH;
    static constexpr bool kPair = sizeof(OUT) == 4, kPages16 = PAGES16;
    // Where row tiles outnumber the workgroups: even pieces in rounds (below), 202 us and not 234 for 64 requests of 512-4096 keys and 128 heads,
    // 224 and not 342 for 100 of 30-3000.  Rows of 256 + 32 pass the cache at half the bytes: there the cut line stays, 92 us and not 99.
    static constexpr bool kEven = KH >= 512;
    static constexpr int kM = 64, kKeys = 64, kBlockThreads = 256, kWaves = 4, kPerUnit = 1, kItemCost = 2, kMinShare = kItemCost + 1;
    static constexpr int kHeadAt = 0, kTailAt = kKeys * KH * 2, kBuf = kTailAt + kKeys * KT * 2;
    typedef OUT Out;
};

// A wave's loads of a tile: rows 16 wave .. 16 wave + 15.  Where they lie is fetched a tile ahead.
//
// A wave that has a SIMD to itself issues an instruction every 4 cycles, eight to a product; of the 18 loads, each with an address and a
// place in LDS of its own, as little as possible is to be computed.  16 consecutive keys of a page are 16 consecutive rows: one page
// number for all of the wave's rows, and addresses that are a scalar plus a lane's constant.
template <class C>
struct LatentLoads {
    typedef RowLoads<C::kHead / 8, C::kWaves> Head;
    typedef RowLoads<C::kTail / 8, C::kWaves> Tail;
    static constexpr int kEach = Head::kEach + Tail::kEach;
    int page, place;      // pages of 16: of the wave's first row (place: behind that row of the page); else of the lane's key
    Buffer from;          // the wave's rows
    uint32_t slot;
    int head_xor, head_add, tail_at;

    __device__ __forceinline__ void place_lane(const Args& a, int lane) {
        constexpr int CH = C::kHead / 8, CT = C::kTail / 8;
        head_xor = ((lane % CH) ^ permutation<CH>(lane / CH)) << 4;
        head_add = (lane / CH) * (int)a.head_stride;
        tail_at = (lane / CT) * (int)a.head_stride + C::kHead * 2 + (((lane % CT) ^ permutation<CT>(lane / CT)) << 4);
    }
    __device__ __forceinline__ void find(const Args& a, const Piece& p, int t, int wave, int lane) {
        if constexpr (C::kPages16) {
            const int key = min(t * C::kKeys + 16 * wave, (p.q.k_end - 1) & ~15);
            const int pg = a.p_shift >= 0 ? key >> a.p_shift : (int)((uint32_t)key / (uint32_t)a.P);
            page = a.bt[(size_t)p.q.table * a.max_pages + pg];
            place = key - pg * a.P;
        } else {
            const Where x = find_key<kLatent>(a, p.q, min(t * C::kKeys + lane, p.q.k_end - 1));
            page = x.page;
            place = (int)x.place;
        }
    }
    // The loads to come are those of the tile that has been found.
    __device__ __forceinline__ void take(const Args& a) {
        if constexpr (C::kPages16)
            from = buffer_at(a.k_head + ((uint64_t)(uint32_t)clamp_to(uniform(page), 0, a.n_pages - 1) * a.page_slots + uniform(place)) * a.head_stride, 16 * a.head_stride);
        else slot = slot_of<kLatent>(a, Where{page, (uint32_t)place});
    }
    // Load i of 16 rows that follow each other in memory.  ENDS: some may be behind the last row (then all of the offset is the lane's: that
    // is what is held against the descriptor).
    template <bool ENDS>
    __device__ __forceinline__ void issue_rows(int i, Buffer rows, int stride, char* buf, int wave) const {
        const bool head = i < Head::kEach;
        const int k = head ? i * Head::kRows : (i - Head::kEach) * Tail::kRows, lane_at = head ? (head_xor ^ ((k & 7) << 5)) + head_add : tail_at;
        to_lds(rows, ENDS ? lane_at + k * stride : lane_at, ENDS ? 0 : k * stride, buf + (head ? C::kHeadAt + (16 * wave + k) * C::kHead * 2 : C::kTailAt + (16 * wave + k) * C::kTail * 2));
    }
    __device__ __forceinline__ void issue(int i, const Args& a, char* buf, int wave, int lane) const {
        if constexpr (C::kPages16) issue_rows<false>(i, from, (int)a.head_stride, buf, wave);
        else if (i < Head::kEach) Head::issue(i, a.k_head, a.head_stride, slot, buf + C::kHeadAt, wave, lane);
        else Tail::issue(i - Head::kEach, a.k_tail, a.tail_stride, slot, buf + C::kTailAt, wave, lane);
    }
};

struct LatentShared {     // what the waves of a workgroup tell each other
    uint16_t p[64][64];   // weights [row][key], 16-byte chunks of a row permuted
    float top[4][32];     // largest product of a row among a wave's keys; at the end its sum of weights
    Reference of[2][32];  // at the end: what the rows' weights refer to
    // By wave.  A tile that take_tile gives up is taken by take_any_tile without a barrier between: another wave may still be reading `ahead`
    // when this one writes again, so that each has flags of its own.
    int ahead[4];         // take_tile: a score is ahead of its reference
    int odd[4];           // take_any_tile: scores that are not finite
    int far[4];           // take_any_tile: references that are no powers of two
};

template <class C>
struct LatentRows {
    static constexpr int kHeadSteps = C::kHead / 16, kTailSteps = C::kTail / 16, kBlocks = C::kDv / 64;  // (half the columns)
    bf16x8 q[kHeadSteps + kTailSteps];
    f32x16 acc[kBlocks];
    Reference of;
    float l;
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

// The sums' place is the accumulation registers.  Where something else than a product touches them, once in many tiles, the compiler would
// otherwise take them to the other registers for all of the loop around it, 256 moves a tile.  change(x) is applied to every element; the
// wait states are those behind a product of 8 passes, and in front of the next.
template <class Change>
__device__ __forceinline__ void change_sums(f32x16& acc, Change change) {
    asm volatile("s_nop 15\n\ts_nop 7" : "+a"(acc));
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        float x, y = acc[e];
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(y));
        x = change(x, e);
        asm volatile("v_accvgpr_write_b32 %0, %1" : "=a"(y) : "v"(x));
        acc[e] = y;
    }
    asm volatile("s_nop 7" : "+a"(acc));
}

// Scores of the wave's 32 keys.
template <class C, class Beside>
__device__ __forceinline__ f32x16 scores_of(const LatentRows<C>& w, const char* buf, Beside beside) {
    typedef LatentRows<C> R;
    return first_product<R::kHeadSteps + R::kTailSteps>([&](int s) __attribute__((always_inline)) {
        return *reinterpret_cast<const bf16x8*>(s < R::kHeadSteps ? buf + C::kHeadAt + w.k_at[s % 8] + (s / 8) * 256 : buf + C::kTailAt + w.tail_at[s - R::kHeadSteps]);
    }, w.q, beside);
}

constexpr float kLeast = 1.17549435e-38f;  // 2^-126, in bf16 as well

template <class C>
__device__ __forceinline__ void write_weights(const LatentRows<C>& w, char* p, const f32x16& z) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
        *reinterpret_cast<u32x2*>(p + w.p_write[k]) = u32x2{bf16_pair(z[4 * k], z[4 * k + 1]), bf16_pair(z[4 * k + 2], z[4 * k + 3])};
}
__device__ __forceinline__ void take_bf16_off(f32x16& z) {
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] -= (float)(__bf16)z[e];
}

// Operand of the second product: keys 16 s + 8 h .. of columns 32 b .. of the wave's half.  (Keys 4 .. 7 of eight: the permutation of
// their rows differs in the bit that tells apart blocks b and b ^ 2.)
template <class C>
__device__ __forceinline__ s16x8 values_of(const LatentRows<C>& w, const char* buf, int s, int b) {
    constexpr int kRow = C::kHead * 2;
    const char* at = buf + C::kHeadAt + 16 * s * kRow + (b / 4) * 256;
    return transposed(at + w.v_at[b % 4], at + 4 * kRow + w.v_at[(b % 4) ^ 2]);
}

// acc += V^T P^T for the wave's half of the columns.
template <class C>
__device__ __forceinline__ void second_product(LatentRows<C>& w, const char* buf, const char* p) {
    typedef LatentRows<C> R;
    bf16x8 weights[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) weights[s] = *reinterpret_cast<const bf16x8*>(p + w.p_read[s]);
    constexpr int kBlocks = R::kBlocks;
    in_turn<4 * kBlocks, 6, s16x8>([&](int k) __attribute__((always_inline)) { return values_of<C>(w, buf, k / kBlocks, k % kBlocks); },
                                   [&](int k, s16x8 v) __attribute__((always_inline)) {
                                       w.acc[k % kBlocks] = product(__builtin_bit_cast(bf16x8, v), weights[k / kBlocks], w.acc[k % kBlocks]);
                                   },
                                   [](int) {});
}
// The same where values are not finite among masked ones: such a value must not meet the zero weight of a row that does not see it.
// Each kind is multiplied as 1 and takes its place only in rows that give it weight.
template <class C>
__device__ __forceinline__ void second_product_carefully(LatentRows<C>& w, const char* buf, const char* p) {
    typedef LatentRows<C> R;
    bf16x8 weights[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) weights[s] = *reinterpret_cast<const bf16x8*>(p + w.p_read[s]);
#pragma unroll
    for (int b = 0; b < R::kBlocks; ++b) {
#pragma unroll
        for (int s = 0; s < 4; ++s) w.acc[b] = product(elements(values_of<C>(w, buf, s, b), kFinite), weights[s], w.acc[b]);
#pragma unroll 1
        for (int kind = kUp; kind <= kNan; ++kind) {
            f32x16 t = zeros();
#pragma unroll
            for (int s = 0; s < 4; ++s) t = product(elements(values_of<C>(w, buf, s, b), kind), weights[s], t);
            const float value = odd_value(kind);
            change_sums(w.acc[b], [&](float x, int e) { return t[e] != 0.0f ? x + value : x; });
        }
    }
}

// A tile of 64 keys that every row sees whole, by references in powers of two.  True: a score is ahead of its row's reference, and nothing
// has been added.  All waves pass the same barriers; those without rows (not `live`) do no more.
// beside(i) issues the wave's load i of the next tile: between the products, whose issue leaves time for it.
template <class C, class Beside>
__device__ __forceinline__ bool take_tile(LatentRows<C>& w, const char* buf, LatentShared& sh, bool live, float scale_log2, int lane, int wave, Beside beside) {
    constexpr int kLoads = LatentLoads<C>::kEach, kSteps = LatentRows<C>::kHeadSteps + LatentRows<C>::kTailSteps;
    static_assert(2 * kLoads <= kSteps, "a load beside every other product");
    char* p = reinterpret_cast<char*>(sh.p);
    f32x16 z;
    float sum = 0.0f;
    bool ahead = false;
    if (live) {
        z = scores_of<C>(w, buf, [&](int s) __attribute__((always_inline)) {
            if (s % 2 == 0 && s / 2 < kLoads) beside(s / 2);
        });
        ahead = __any(largest(z) * scale_log2 > w.of.log2);
        sum = weights_of(z, Reference{0.0f, w.of.log2}, scale_log2);
        write_weights<C>(w, p, z);
    } else {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) beside(i);
    }
    if (lane == 0) sh.ahead[wave] = ahead;
    lds_barrier();
    if (uniform(sh.ahead[0] | sh.ahead[1] | sh.ahead[2] | sh.ahead[3])) return true;
    if (live) {
        w.l += sum;
        second_product<C>(w, buf, p);
    }
    if constexpr (C::kPair) {
        lds_barrier();
        if (live) {
            take_bf16_off(z);
            write_weights<C>(w, p, z);
        }
        lds_barrier();
        if (live) second_product<C>(w, buf, p);
    }
    return false;
}

// Any tile: some keys may be masked, references move if they have to.  (Rows that see none of its keys give zero weights.)  True: all of the
// workgroup's references are powers of two.
template <class C>
__device__ __forceinline__ bool take_any_tile(LatentRows<C>& w, const char* buf, LatentShared& sh, int key0, bool live, float scale_log2, int lane, int wave) {
    const int li = lane & 31, h = lane >> 5, part = wave & 1;
    char* p = reinterpret_cast<char*>(sh.p);
    f32x16 z;
    float top = -INFINITY;
    int odd_scores = 0;
    if (live) {
        z = scores_of<C>(w, buf, [](int) {});
        float odd = 0.0f;  // a value that is not finite is in its key, too, and has made the key's scores infinite or NaN
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            odd += z[e] - z[e];
            z[e] = key0 + 32 * part + 8 * (e >> 2) + 4 * h + (e & 3) <= w.seen ? z[e] : -INFINITY;
        }
        odd_scores = __any(odd != 0.0f);
        top = largest(z);
    }
    if (h == 0) sh.top[wave][li] = top;
    if (lane == 0) sh.odd[wave] = odd_scores;
    lds_barrier();
    const bool careful = uniform(sh.odd[wave & 2] | sh.odd[wave | 1]);
    if (live) {
        const float both = fmaxf(sh.top[wave & 2][li], sh.top[wave | 1][li]);
        const Reference old = w.of;
        const bool ahead = exponent(both, old, scale_log2) > 0.0f, moved = ahead && old.log2 > -INFINITY;
        if (ahead) w.of = reference_for(both, scale_log2);
        if (__any(moved)) {
            const float alpha = moved ? __builtin_amdgcn_exp2f(distance(old, w.of, scale_log2)) : 1.0f;
            w.l *= alpha;
#pragma unroll
            for (int b = 0; b < LatentRows<C>::kBlocks; ++b) change_sums(w.acc[b], [&](float x, int) { return x * alpha; });
        }
        w.l += weights_of(z, w.of, scale_log2);
        if (careful)  // a value that is not finite reaches every row that sees it, however small the weight
#pragma unroll
            for (int e = 0; e < 16; ++e) z[e] = key0 + 32 * part + 8 * (e >> 2) + 4 * h + (e & 3) <= w.seen && z[e] < kLeast ? kLeast : z[e];
        write_weights<C>(w, p, z);
    }
    const int far = live && __any(w.of.raw != 0.0f);
    if (lane == 0) sh.far[wave] = far;
    lds_barrier();
    const bool near = !uniform(sh.far[0] | sh.far[1] | sh.far[2] | sh.far[3]);
    if (live) {
        if (careful) second_product_carefully<C>(w, buf, p);
        else second_product<C>(w, buf, p);
    }
    if constexpr (C::kPair) {  // (where a weight's first part has met a value that is not finite, its rest has nothing to add)
        lds_barrier();
        if (live) {
            take_bf16_off(z);
            write_weights<C>(w, p, z);
        }
        lds_barrier();
        if (live) {
            if (careful) second_product_carefully<C>(w, buf, p);
            else second_product<C>(w, buf, p);
        }
    }
    return near;
}

template <class C>
__device__ __forceinline__ void run_latent(const Args& a, const Piece& p, char* buf0, char* buf1, LatentShared& sh) {
    typedef LatentRows<C> R;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), li = lane & 31, h = lane >> 5, part = wave & 1;
    const int n_packed = p.q.rows * a.G, first = p.rt * C::kM + (wave >> 1) * 32;
    const bool live = first < n_packed;  // a wave without rows helps to load
    R w;
    w.of = Reference{0.0f, -INFINITY};
    w.l = 0.0f;
    w.seen = -1;
    w.place_operands(lane, wave >> 1, part);
    LatentLoads<C> loads;
    loads.place_lane(a, lane);
    if (live) w.seen = last_key(a, p.q, min(first + li, n_packed - 1));
    const int all_see = last_key(a, p.q, p.rt * C::kM);  // the tile's first row, and with it every row
    int t = p.t0;
    auto load_all = [&](char* to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LatentLoads<C>::kEach; ++i) loads.issue(i, a, to, wave, lane);
    };
    __syncthreads();  // nobody reads the buffers any more
    if (t < p.t1) {
        loads.find(a, p, t, wave, lane);
        // the queries, 64 rows that follow each other and have a key's shape, come by way of the other buffer
        const size_t row0 = (size_t)p.q.row0 * a.H + p.rt * C::kM + 16 * wave, rows = (size_t)a.N_cap * a.H;
        const int stride = (int)a.head_stride;
        const Buffer queries = buffer_at((const char*)a.q + min(row0, rows - 1) * stride, row0 < rows ? (uint32_t)min(rows - row0, (size_t)16) * stride : 0u);
#pragma unroll
        for (int i = 0; i < LatentLoads<C>::kEach; ++i) loads.template issue_rows<true>(i, queries, stride, buf1, wave);
        loads.take(a);
        loads.find(a, p, min(t + 1, p.t1 - 1), wave, lane);
        load_all(buf0);
        arrive();
        const int other = ((wave >> 1) - part) * 32;  // from the wave's keys to its rows
#pragma unroll
        for (int s = 0; s < R::kHeadSteps; ++s) w.q[s] = *reinterpret_cast<const bf16x8*>(buf1 + C::kHeadAt + other * C::kHead * 2 + w.k_at[s % 8] + (s / 8) * 256);
#pragma unroll
        for (int s = 0; s < R::kTailSteps; ++s) w.q[R::kHeadSteps + s] = *reinterpret_cast<const bf16x8*>(buf1 + C::kTailAt + other * C::kTail * 2 + w.tail_at[s]);
    }
    u32x4 none = {0, 0, 0, 0};
#pragma unroll
    for (int b = 0; b < R::kBlocks; ++b) {  // zeros by a product each: one instruction where 16 registers would be set
        asm volatile("" : "+v"(none));
        w.acc[b] = product(__builtin_bit_cast(bf16x8, none), __builtin_bit_cast(bf16x8, none), zeros());
    }
    auto whole = [&] { return t < p.t1 && p.q.k_begin + t * C::kKeys + C::kKeys - 1 <= all_see; };
    // A tile of the fast loop; false: a reference moves, and the tile is still to be added (the next one's loads are under way).
    auto step = [&](const char* now, char* then) __attribute__((always_inline)) {
        arrive();  // (and nobody reads the other buffer any more)
        loads.take(a);
        loads.find(a, p, min(t + 2, p.t1 - 1), wave, lane);  // (behind the last tile this one is loaded again: a load too many costs less than asking)
        const bool ahead = take_tile<C>(w, now, sh, live, a.scale_log2, lane, wave, [&](int i) __attribute__((always_inline)) { loads.issue(i, a, then, wave, lane); });
        t += !ahead;
        return !ahead;
    };
    bool loaded = false;  // the next tile's loads have been issued
    while (t < p.t1) {
        // the first tile, tiles with masked keys, tiles where a reference moves
        const bool odd = (t - p.t0) & 1;
        if (!loaded) {
            arrive();
            loads.take(a);
            loads.find(a, p, min(t + 2, p.t1 - 1), wave, lane);
            load_all(odd ? buf0 : buf1);
        }
        loaded = false;
        const bool near = take_any_tile<C>(w, odd ? buf1 : buf0, sh, p.q.k_begin + t * C::kKeys, live, a.scale_log2, lane, wave);
        ++t;
        // all the others: here the sums are the matrix instructions' alone, and stay in the accumulation registers
        if (!odd && near) {
            w.of.raw = 0.0f;  // (known, and in no register of the loop)
            while (whole()) {
                if (!step(buf1, buf0)) { loaded = true; break; }
                if (!whole()) break;
                if (!step(buf0, buf1)) { loaded = true; break; }
            }
        }
    }
    // The sums leave by way of LDS, row by row: from the accumulators a store would touch 32 rows.  (16-byte chunks permuted by row, so
    // that eight rows' writes of one column reach all banks.)
    w.l += other_half(w.l);
    arrive();  // (the load too many has its place until it has come)
    if (h == 0) sh.top[wave][li] = w.l;
    if (h == 0 && part == 0) sh.of[wave >> 1][li] = w.of;
    constexpr int kRowBytes = C::kDv * 4;
    static_assert(32 * kRowBytes <= C::kBuf, "32 rows' sums fit into a buffer");
    auto place = [&](int row, int chunk) { return (row < 32 ? buf0 : buf1) + (row & 31) * kRowBytes + ((chunk ^ (row & 7)) << 4); };
#pragma unroll
    for (int b = 0; b < R::kBlocks; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4*>(place((wave >> 1) * 32 + li, part * (C::kDv / 8) + 8 * b + 2 * g + h)) =
                f32x4{w.acc[b][4 * g], w.acc[b][4 * g + 1], w.acc[b][4 * g + 2], w.acc[b][4 * g + 3]};
    __syncthreads();
    const int rows = min(n_packed - p.rt * C::kM, C::kM);
    const size_t row0 = (size_t)p.q.row0 * a.H + p.rt * C::kM, slot0 = (size_t)p.slot * a.m_cap;  // (a request's rows follow each other)
#pragma unroll 1
    for (int r = wave; r < rows; r += C::kWaves) {
        const float l = sh.top[r >> 5 << 1][r & 31] + sh.top[(r >> 5 << 1) | 1][r & 31];
        const Reference of = sh.of[r >> 5][r & 31];
        f32x4 x[C::kDv / 256];
#pragma unroll
        for (int k = 0; k < C::kDv / 256; ++k) x[k] = *reinterpret_cast<const f32x4*>(place(r, k * 64 + lane));
        if (p.whole) {
            const float inv = inverse(l);
#pragma unroll
            for (int k = 0; k < C::kDv / 256; ++k) store4((typename C::Out*)a.out + (row0 + r) * C::kDv + 4 * (k * 64 + lane), x[k] * inv);
            if (lane == 0 && a.lse) a.lse[row0 + r] = log_sum<kLatent>(of, l, a.scale);
        } else {
#pragma unroll
            for (int k = 0; k < C::kDv / 256; ++k) store4(a.part_o + (slot0 + r) * C::kDv + 4 * (k * 64 + lane), x[k]);
            if (lane == 0) store4(a.part_ml + 4 * (slot0 + r), f32x4{of.raw, of.log2, l, 0.0f});
        }
    }
}

// Even pieces: where a batch has no more row tiles than there are workgroups, every item is cut into pieces of about the same length,
// as long as makes one piece for each workgroup: half the sums of a cut line, each workgroup takes up one piece, and pieces of the same
// keys, row tile by row tile, are neighbours (and share a die's cache).  The length is the shortest of 64 candidates, one per lane, from
// an equal share of all key tiles upwards, for which the pieces do not outnumber the workgroups.  Where there are more row tiles, every
// workgroup takes up to kEvenRounds pieces: taking one up costs 38000 cycles (7 tiles), but row tiles of a request that run at different
// keys read these anew from behind the die's cache, 8000 cycles a tile and not 5300.  False: the line is cut instead, where the length that
// is needed is much beyond an equal share: few long requests among as many short ones as there are workgroups.  us by the line / by even
// pieces, 16 heads: within the bound, 32 requests of 1024-8192 keys 82 / 59, one of 8000 and 31 of 100-500 60 / 55, 250 of 300 77 / 51; just
// beyond it, 230 of 500 and 20 of 900 83 / 68, 220 of 300 and 30 of 2000 86 / 98; far beyond it, 240 of 64 and 10 of 8000 95 / 259.
constexpr int kEvenRequests = 256;
struct EvenScratch {
    int tiles[kEvenRequests], row_tiles[kEvenRequests];
    int counts[4][kWave];
    int sums[8];
    int piece[8];
};
template <class C>
__device__ __forceinline__ bool even_piece(const Args& a, int share, EvenScratch& x, Piece& p, bool& mine, int& rounds) {
    static_assert(C::kBlockThreads == kEvenRequests && C::kWaves == 4, "a request per thread");
    if (a.B > kEvenRequests) return false;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    Seq q{};
    int nk = 0, nrt = 0;
    if (tid < a.B) {
        q = sequence<C::kOp>(a, tid);
        nrt = row_tiles_of<C>(a, q);
        nk = nrt ? key_tiles<C>(a, q, 0) : 0;
    }
    x.tiles[tid] = nk;
    x.row_tiles[tid] = nrt;
    const int tiles = wave_sum_i(min(nk, 1 << 20) * min(nrt, 1 << 10)), items = wave_sum_i(nrt);
    if (lane == 0) {
        x.sums[wave] = tiles;
        x.sums[4 + wave] = items;
    }
    __syncthreads();
    const int n_items = uniform((x.sums[4] + x.sums[5]) + (x.sums[6] + x.sums[7]));
    const int most = n_items <= a.nb ? a.nb : a.even_cap;  // pieces
    if (n_items > most || n_items == 0) return false;
    rounds = most == a.nb ? 1 : kEvenRounds;
    const int n_tiles = uniform((x.sums[0] + x.sums[1]) + (x.sums[2] + x.sums[3]));
    // Where workgroups are plenty: a tile more of a piece takes 2 us, a piece more of a join a sixth of that.  Length l of t tiles costs
    // 2 l + t / 3 l, least at sqrt(t / 6).  (8000 keys, 16 heads: 69 us in 126 pieces of one tile, 47 us in 27.)
    const int cheapest = (int)(__builtin_amdgcn_sqrtf((float)n_tiles * __builtin_amdgcn_rcpf(6.0f * n_items)) + 0.5f);
    const int shortest = max(max(cheapest, 1), ceil_div(n_tiles, most));
    const int length = lane == 63 ? 1 << 24 : shortest + ((shortest * lane + 15) >> 4);
    const float inv = 1.0f / (float)length;
    auto pieces_of = [&](int tiles, int length, float inv) {  // ceil(tiles / length), at least 1
        int n = max((int)((float)tiles * inv), 1);
        n += n * length < tiles;
        return n + (n * length < tiles);
    };
    int count = 0;
#pragma unroll 1
    for (int i = wave; i < a.B; i += 4) count += x.row_tiles[i] * pieces_of(x.tiles[i], length, inv);
    x.counts[wave][lane] = count;
    __syncthreads();
    count = (x.counts[0][lane] + x.counts[1][lane]) + (x.counts[2][lane] + x.counts[3][lane]);
    const int pick = __ffsll((unsigned long long)__ballot(count <= most)) - 1;  // (lane 63 cuts nothing)
    const int chosen = __builtin_amdgcn_readlane(length, pick);
    if (chosen > shortest + (shortest >> 2) + 3) return false;  // lengths too uneven for that
    const int pieces = nrt ? pieces_of(nk, chosen, 1.0f / (float)chosen) : 0;
    int upto = wave_inclusive_scan_dpp(nrt * pieces);
    if (lane == 63) x.sums[wave] = upto;
    __syncthreads();
    for (int k = 0; k < wave; ++k) upto += x.sums[k];
    const int begin = upto - nrt * pieces;
    if (tid == 0) x.piece[0] = 0;
    __syncthreads();
    if (share >= begin && share < upto) {
        x.piece[0] = pieces;
        x.piece[1] = share - begin;
        x.piece[2] = q.row0;
        x.piece[3] = q.rows;
        x.piece[4] = q.k_end;
        x.piece[5] = q.base;
        x.piece[6] = tid;
        x.piece[7] = nk;
    }
    __syncthreads();
    int32_t* desc = a.desc + (size_t)share * kDescInts;
    p.pieces = uniform(x.piece[0]);
    mine = p.pieces > 0;
    if (!mine) {
        if (tid == 0) desc[0] = 0;
        return true;
    }
    p.q.row0 = uniform(x.piece[2]);
    p.q.rows = uniform(x.piece[3]);
    p.q.k_begin = 0;
    p.q.k_end = uniform(x.piece[4]);
    p.q.base = uniform(x.piece[5]);
    p.q.table = uniform(x.piece[6]);
    p.q.first = 0;
    const int at = uniform(x.piece[1]), all = uniform(x.piece[7]), tiles_of_rows = row_tiles_of<C>(a, p.q);
    const int which = (int)((uint32_t)at / (uint32_t)tiles_of_rows), each = (int)((uint32_t)all / (uint32_t)p.pieces), longer = all - each * p.pieces;
    p.hk = 0;
    p.rt = at - which * tiles_of_rows;
    p.t0 = which * each + min(which, longer);
    p.t1 = p.t0 + each + (which < longer);
    p.whole = p.pieces == 1;
    p.slot = share;
    p.share0 = share;
    if (tid == 0) {
        const bool first = which == 0 && !p.whole;
        desc[1] = p.q.row0; desc[2] = 0; desc[3] = p.rt; desc[4] = min(p.q.rows * a.G - p.rt * C::kM, C::kM);
        desc[5] = p.slot; desc[6] = p.slot + tiles_of_rows; desc[7] = tiles_of_rows;
        desc[0] = first ? p.pieces : 0;
    }
    return true;
}

template <class C>
__global__ __launch_bounds__(C::kBlockThreads, 1) void latent_kernel(Args a) {
    __shared__ __align__(1024) char buf0[C::kBuf];
    __shared__ __align__(1024) char buf1[C::kBuf];
    __shared__ __align__(1024) LatentShared sh;
    const int share = share_of_block(blockIdx.x, a.nb);
    Piece p;
    Walk<C> walk;
    bool more = false, even = true;
    int round = 0, rounds = 1;
    if (threadIdx.x == 0)
        for (int k = share + a.nb; k < a.even_cap; k += a.nb) a.desc[(size_t)k * kDescInts] = 0;
    for (;;) {
        if (even) {
            __syncthreads();  // nobody reads the buffers any more
            even = even_piece<C>(a, share + round * a.nb, *reinterpret_cast<EvenScratch*>(buf1), p, more, rounds);
            if (!even) walk.begin(a, share, find_share<C>(a, share, reinterpret_cast<long long*>(buf0)));
        }
        if (!even) more = walk.next(a, share, p);
        if (more) run_latent<C>(a, p, buf0, buf1, sh);
        if (even ? ++round == rounds : !more) break;
    }
}
template <int KH, int KT, class OUT, bool PAGES16>
struct Kernel<Latent<KH, KT, OUT, PAGES16>> {
    static constexpr auto run = latent_kernel<Latent<KH, KT, OUT, PAGES16>>;
};

}  // namespace row_tiles
}  // namespace fsr
