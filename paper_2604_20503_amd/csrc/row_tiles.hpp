// Attention of many query rows on one stream of keys: what attention over a latent cache, its expanded form, attention
// behind a shared prefix and attention of trees have in common.
//
// A *sequence* is a set of query rows that read the same keys (a request's rows, or all rows of the requests that share a
// prefix); per stream head, G query heads of a call row read the same key.  The rows of a sequence are packed (packed row r =
// call row r / G, query head r % G of the stream head) and cut into tiles of M rows; an *item* is one tile with all its keys.
//     z[r, t] = scale * q[r] . k[t],   o[r] = sum_t exp(z[r, t] - m) v[t] / sum_t exp(z[r, t] - m)
//
// Schedule: the key tiles of all items lie end to end on a line (every item with C::kItemCost units in front for taking it up),
// and the line is cut into equal shares, one per workgroup of a persistent grid.  Lengths stay on the device: every workgroup
// adds them up for itself.  An item inside one share is finished there; one that a share boundary cuts leaves unnormalised
// fp32 sums of its pieces in the workspace, at most two per share, which a second launch adds in the order of the shares
// (no atomics: results do not depend on timing).
#pragma once
#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "common.hpp"
#include "device_utils.hpp"

namespace fsr {
namespace row_tiles {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
typedef __attribute__((__vector_size__(8 * sizeof(short)))) short s16x8;
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kThreads = 256;      // of the kernels below, where a configuration does not say otherwise
constexpr int kWaves = kThreads / kWave;
constexpr int kTileRows = 128;     // most rows of a tile
constexpr int kDescInts = 8;       // merge descriptor of a share
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kSharesCap = 512;
constexpr int kMaxBlocks = 1 << 23;  // of a launch: its threads are counted in 32 bits
constexpr int kEvenRounds = 3;       // latent: most pieces of a workgroup in a batch that is cut evenly
constexpr int kRefPlace = 10, kRefPrefix = 1 << 24;  // fields of a reference to a part of a row: its place in the tile; there is a prefix before it
constexpr float kAhead = 40.0f;    // distance of a row's exponent reference from its largest score, in powers of two

enum : int { kLatent = 0, kExpanded = 1, kShared = 2, kTree = 3 };

struct Args {
    const void* q;       // [N_cap, H, D_k]
    const char* k_head;  // first (or only) part of a key row
    const char* k_tail;  // rest of a key row
    const char* v;       // value row (latent: the first part of the key row)
    const int32_t* bt;
    const int32_t* ctx;
    const int32_t* cu_q;
    const int32_t* cu_k;      // expanded: offsets of the keys
    const int32_t* cu_groups; // shared
    const int32_t* prefix;    // shared
    const uint32_t* tree;     // tree: [N_cap][tree_words] the rows of its request that a row sees, a bit each
    int tree_words;
    void* out;
    float* lse;
    int B, N_cap, H, H_stream, G, n_groups, T_cap;
    int P, p_shift, max_pages, n_pages;  // p_shift: log2(P), or -1 if P is no power of two
    uint32_t page_slots;                    // slots that a page advances by
    uint32_t head_stride, tail_stride, v_stride;   // bytes from a slot to the next
    long long head_hk, v_hk;                // bytes from a stream head to the next
    float scale, scale_log2;  // softmax scale, and times log2(e)
    int nb, shares_cap, min_share, m_cap;
    int even_cap;     // latent: most pieces of a batch that is cut evenly
    float* part_o;    // [2 * shares_cap][m_cap][D_v]
    float* part_ml;   // [2 * shares_cap][m_cap][4] what the weights refer to (a Reference), their sum
    int32_t* desc;    // [2 * shares_cap][kDescInts]
    float* row_o;     // shared: [2][N_cap * H][D_v] sums of items that are whole: prefix, own
    float* row_ml;    // shared: [2][N_cap * H][4]
    int32_t* refs;    // shared: [2][N_cap * H][2] pieces of the item (0: in row_o; -1: done); its first share, the row's place in its tile, kRefPrefix
};

struct Seq {
    int row0, rows;      // call rows
    int k_begin, k_end;  // keys (tiles begin at k_begin)
    int k_first;         // the first one that is seen
    int base;            // packed row r sees keys up to base + r / G (tree: the keys in front of base, and of the others what its bits say)
    int table;           // row of the block table
    uint32_t first;      // expanded: slot of the first key
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ int clamp_to(int x, int lo, int hi) { return min(max(x, lo), hi); }

template <int OP>
__device__ __forceinline__ int n_sequences(const Args& a) { return OP == kShared ? a.n_groups + a.B : a.B; }

// Sequence s.  Metadata that does not hold together (offsets out of order, lengths beyond the table) never leads outside the
// tensors: offsets are clamped to the rows that are allocated, positions to the table.
template <int OP>
__device__ __forceinline__ Seq sequence(const Args& a, int s) {
    Seq q;
    q.first = 0;
    q.k_first = 0;
    if constexpr (OP == kExpanded) {
        q.row0 = clamp_to(a.cu_q[s], 0, a.N_cap);
        q.rows = clamp_to(a.cu_q[s + 1], q.row0, a.N_cap) - q.row0;
        const int first = clamp_to(a.cu_k[s], 0, a.T_cap);
        const int keys = clamp_to(a.cu_k[s + 1], first, a.T_cap) - first;
        q.first = (uint32_t)first;
        q.k_begin = 0;
        q.k_end = keys;
        q.base = keys - q.rows;
        q.table = 0;
        return q;
    }
    const int cap = (int)min((long long)a.max_pages * a.P, 1LL << 30);
    if (OP == kShared && s < a.n_groups) {
        const int i0 = clamp_to(a.cu_groups[s], 0, a.B), i1 = clamp_to(a.cu_groups[s + 1], i0, a.B);
        q.row0 = clamp_to(a.cu_q[i0], 0, a.N_cap);
        q.rows = clamp_to(a.cu_q[i1], q.row0, a.N_cap) - q.row0;
        q.k_begin = 0;
        q.k_end = i1 > i0 ? clamp_to(a.prefix[s], 0, cap) : 0;
        if (q.k_end == 0) q.rows = 0;  // no item: the rows are their own part's alone
        q.base = 1 << 30;              // every row sees the whole prefix
        q.table = min(i0, a.B - 1);
        return q;
    }
    const int i = OP == kShared ? s - a.n_groups : s;
    q.row0 = clamp_to(a.cu_q[i], 0, a.N_cap);
    q.rows = clamp_to(a.cu_q[i + 1], q.row0, a.N_cap) - q.row0;
    q.k_begin = 0;
    if constexpr (OP == kShared) {
        int lo = 0, hi = a.n_groups;  // the group that holds request i
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.cu_groups[mid] <= i) lo = mid; else hi = mid;
        }
        const bool in = a.cu_groups[lo] <= i && i < a.cu_groups[lo + 1];
        q.k_first = in ? clamp_to(a.prefix[lo], 0, cap) : 0;
        q.k_begin = q.k_first & ~15;  // (16 rows of a tile lie in one page, if pages hold a multiple of 16 tokens)
        if (!in) q.rows = 0;  // requests outside the groups have no output
    }
    const int c = clamp_to(a.ctx[i], q.k_first, cap);
    q.base = c;
    q.k_end = min(c + min(q.rows, cap), cap);
    q.table = i;
    return q;
}

__device__ __forceinline__ int ceil_div(int x, int y) { return (int)((uint32_t)(x + y - 1) / (uint32_t)y); }  // 0 <= x, 0 < y

template <class C>
__device__ __forceinline__ int row_tiles_of(const Args& a, const Seq& q) {
    return ceil_div(q.rows * a.G, C::kM);
}

// Key tiles of row tile rt.
template <class C>
__device__ __forceinline__ int key_tiles(const Args& a, const Seq& q, int rt) {
    int end = q.k_end;
    if constexpr (C::kOp == kExpanded) end = min(end, q.base + min(q.rows, (rt + 1) * C::kM));  // (G = 1) the last row's last key
    return end > q.k_first ? ceil_div(end - q.k_begin, C::kKeys) : 0;
}

// Units of the line in front of row tile rt of a stream head.
template <class C>
__device__ __forceinline__ long long units_before(const Args& a, const Seq& q, int rt) {
    if constexpr (C::kOp != kExpanded) return (long long)rt * (C::kItemCost + key_tiles<C>(a, q, 0));
    // expanded: key_tiles grows by M / kKeys per row tile from the first tile that sees a key, except that the last tile may
    // hold fewer rows (it is summed by itself)
    static_assert(C::kOp != kExpanded || C::kM % C::kKeys == 0, "whole key tiles per row tile");
    constexpr int kStep = C::kM / C::kKeys;
    const int n = row_tiles_of<C>(a, q);
    const int full = min(rt, max(n - 1, 0));
    const int t0 = q.base >= 0 ? ceil_div(q.base, C::kKeys) : -((-q.base) / C::kKeys);  // ceil(base / kKeys)
    // tiles r in [r0, full) see t0 + kStep * (r + 1) key tiles
    const int r0 = t0 >= -kStep + 1 ? 0 : min((-t0) / kStep, full);
    const long long m = full - r0;
    long long sum = m * t0 + (long long)kStep * (m * (r0 + 1) + m * (m - 1) / 2);
    sum += (long long)C::kItemCost * full;
    if (rt > full) sum += C::kItemCost + key_tiles<C>(a, q, n - 1);
    return sum;
}

template <class C>
__device__ __forceinline__ long long sequence_units(const Args& a, const Seq& q) {
    return units_before<C>(a, q, row_tiles_of<C>(a, q)) * a.H_stream;
}

// Units are 64-bit numbers below 2^53: a quotient is taken in fp64 and put right where it is one off.
__device__ __forceinline__ long long quotient(long long x, long long y) {
    long long q = (long long)((double)x / (double)y);
    q -= q * y > x;
    return q + ((q + 1) * y <= x);
}

struct Line {
    long long each;        // units of a share, one more in the first `longer` shares
    int longer, shares;
    int seq;               // sequence in which this share begins
    long long seq_start;   // its first unit
    long long lo, hi;      // this share
    bool known;            // `first` is that sequence
    Seq first;
    __device__ __forceinline__ long long begin(int s) const { return each * s + min(s, longer); }
    __device__ __forceinline__ int share_of(long long u) const {
        const long long head = (each + 1) * longer;
        return (int)(u < head ? quotient(u, each + 1) : longer + quotient(u - head, each));
    }
};

__device__ __forceinline__ long long shfl_up64(long long v, int d) {
    const int lo = __shfl_up((int)(uint32_t)v, d, kWave), hi = __shfl_up((int)(v >> 32), d, kWave);
    return ((long long)hi << 32) | (uint32_t)lo;
}

// The share of a line whose units have been added up, `total`; the sequence in which it begins is still to be found.
template <class C>
__device__ __forceinline__ Line cut_line(const Args& a, int share, long long total, int n) {
    Line l;
    l.shares = (int)max(1LL, min((long long)a.nb, quotient(total, a.min_share)));
    l.each = quotient(total, l.shares);
    l.longer = (int)(total - l.each * l.shares);
    l.seq = n;
    l.seq_start = total;
    l.lo = l.hi = 0;
    l.known = false;
    if (total > 0 && share < l.shares) {
        l.lo = l.begin(share);
        l.hi = l.begin(share + 1);
    }
    return l;
}

// Trees of up to 64 requests: a request a lane, every wave for itself, without LDS and barriers (5700 -> 3400 cycles at the start of a call).
template <class C>
__device__ __forceinline__ Line find_share_by_wave(const Args& a, int share) {
    const int n = n_sequences<C::kOp>(a), lane = threadIdx.x & (kWave - 1);
    const Seq q = sequence<C::kOp>(a, min(lane, n - 1));
    long long upto = lane < n ? sequence_units<C>(a, q) : 0;
    const long long mine = upto;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const long long up = shfl_up64(upto, o);
        if (lane >= o) upto += up;
    }
    auto of_lane = [&](long long v, int at) { return (long long)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), at) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, at); };
    Line l = cut_line<C>(a, share, of_lane(upto, kWave - 1), n);
    if (l.lo < l.hi) {
        l.seq = __popcll(__ballot(upto <= l.lo));  // (those that end in front of the share)
        l.seq_start = of_lane(upto - mine, l.seq);
        l.known = true;
        l.first = q;
        l.first.row0 = __builtin_amdgcn_readlane(q.row0, l.seq);
        l.first.rows = __builtin_amdgcn_readlane(q.rows, l.seq);
        l.first.k_end = __builtin_amdgcn_readlane(q.k_end, l.seq);
        l.first.base = __builtin_amdgcn_readlane(q.base, l.seq);
        l.first.table = l.seq;
    }
    return l;
}

// Adds up the line; `scratch`: LDS for C::kBlockThreads sums and one sum per wave.
template <class C>
__device__ __forceinline__ Line find_share(const Args& a, int share, long long* scratch) {
    const int n = n_sequences<C::kOp>(a), tid = threadIdx.x;
    const int each = ceil_div(n, C::kBlockThreads);
    const int s0 = min(tid * each, n), s1 = min(s0 + each, n);
    long long mine = 0;
    for (int s = s0; s < s1; ++s) mine += sequence_units<C>(a, sequence<C::kOp>(a, s));
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const long long up = shfl_up64(upto, o);
        if ((tid & (kWave - 1)) >= o) upto += up;
    }
    if ((tid & (kWave - 1)) == kWave - 1) scratch[C::kBlockThreads + (tid >> 6)] = upto;
    __syncthreads();
    for (int w = 0; w < (tid >> 6); ++w) upto += scratch[C::kBlockThreads + w];
    scratch[tid] = upto;
    __syncthreads();
    Line l = cut_line<C>(a, share, scratch[C::kBlockThreads - 1], n);
    if (l.lo < l.hi) {
        int first = 0, last = C::kBlockThreads - 1;  // the chunk of sequences that holds unit lo
        while (first < last) {
            const int mid = (first + last) >> 1;
            if (scratch[mid] <= l.lo) first = mid + 1; else last = mid;
        }
        first = uniform(first);
        long long at = first ? scratch[first - 1] : 0;
        for (int s = first * each; s < n; ++s) {
            const long long u = sequence_units<C>(a, sequence<C::kOp>(a, s));
            if (at + u > l.lo) {
                l.seq = s;
                l.seq_start = at;
                break;
            }
            at += u;
        }
    }
    __syncthreads();  // the scratch memory is given back
    return l;
}

// The piece of an item that a workgroup works on.
struct Piece {
    Seq q;
    int hk, rt;
    int t0, t1;          // its key tiles
    bool whole;          // all of the item's tiles
    int slot;            // of the partial sums of a piece that is not
    int share0, pieces;  // where the item's pieces lie
};

// Where the packed row r of an item goes.
struct Place {
    int row, head;
};
__device__ __forceinline__ Place place_of(const Args& a, int row0, int hk, int r) {
    const int j = (int)((uint32_t)r / (uint32_t)a.G);
    return Place{row0 + j, hk * a.G + (r - j * a.G)};
}

// Where a key of a sequence lies: its page as the table has it (fetched ahead of use) and its place there.
struct Where {
    int page;
    uint32_t place;
};
template <int OP>
__device__ __forceinline__ Where find_key(const Args& a, const Seq& q, int key) {
    if constexpr (OP == kExpanded) return Where{0, q.first + (uint32_t)key};
    const uint32_t pg = a.p_shift >= 0 ? (uint32_t)key >> a.p_shift : (uint32_t)key / (uint32_t)a.P;
    return Where{a.bt[(size_t)q.table * a.max_pages + pg], (uint32_t)key - pg * (uint32_t)a.P};
}
template <int OP>
__device__ __forceinline__ uint32_t slot_of(const Args& a, Where w) {  // (inside the pool whatever the table holds)
    if constexpr (OP == kExpanded) return w.place;
    return (uint32_t)clamp_to(w.page, 0, a.n_pages - 1) * a.page_slots + w.place;
}

__device__ __forceinline__ uint32_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ uint32_t bf16_pair(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((__attribute__((ext_vector_type(2))) float){x, y}, __attribute__((ext_vector_type(2))) __bf16));
}

// D_v columns of a row: out of the accumulators of one lane, four neighbouring columns at a time.
__device__ __forceinline__ void store4(float* p, f32x4 x) { *reinterpret_cast<f32x4*>(p) = x; }
__device__ __forceinline__ void store4(uint16_t* p, f32x4 x) {
    *reinterpret_cast<u32x2*>(p) = u32x2{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
}

// What a row's weights refer to: product z weighs 2^((z - raw) * scale_log2 - log2).  One of the two numbers would do, were they exact.  In
// powers of two (raw = 0) the exponent is one fma a score, but a reference beyond 2^27 is rounded by more than it is kept ahead: weights would
// overflow, or vanish for a whole row.  There the reference is a product, from which differences are as exact as the products themselves, also
// where their multiples by the scale are beyond fp32.
struct Reference {
    float raw, log2;
};
constexpr float kNear = 134217728.0f;  // 2^27, where a reference's rounding is half a step of 8, and so is its largest score's
__device__ __forceinline__ float exponent(float z, Reference of, float scale_log2) { return fmaf(z - of.raw, scale_log2, -of.log2); }
__device__ __forceinline__ float distance(Reference x, Reference y, float scale_log2) { return fmaf(x.raw - y.raw, scale_log2, x.log2 - y.log2); }  // powers of two
// For a row whose largest product is `top`.
__device__ __forceinline__ Reference reference_for(float top, float scale_log2) {
    const float score = top * scale_log2;
    return fabsf(score) <= kNear ? Reference{0.0f, score + kAhead} : Reference{top, kAhead};
}

// Logarithm of the sum of exp of the scores whose weights add up to l, -inf without any weight.
// (Trees: the powers of two of reference and sum are added first.  A reference is 2^40 ahead, the sum as much smaller, and logarithms of
// that size are off by 2.6e-6 each.)
template <int OP>
__device__ __forceinline__ float log_sum(Reference of, float l, float scale) {
    if constexpr (OP == kTree)
        return l == 0.0f ? -INFINITY : fmaf(of.raw, scale, ((of.log2 + (float)__builtin_amdgcn_frexp_expf(l)) + __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(l))) * kLn2);
    return l == 0.0f ? -INFINITY : fmaf(of.raw, scale, of.log2 * kLn2) + __builtin_amdgcn_logf(l) * kLn2;
}
__device__ __forceinline__ float inverse(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }

typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_at(const char* base, uint32_t bytes) { return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, bytes, 0x00027000); }
// A store that goes past the caches of a die (16: its device-scope bit).  Whole lines of sums that other workgroups read: what lies in a die's
// L2 at a launch's end has to be written from there before the next one starts (28 trees of 5-131 rows, 8/2 heads: 48.3 us, not 45.6).
__device__ __forceinline__ void store_through(Buffer to, int at, f32x4 x) { __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), to, at, 0, 16); }

// Where the result of a row's share of the keys goes.
template <class C>
struct Target {
    typename C::Out* out;  // the result (kDv values and, if wanted, lse), or
    float* lse;
    float* sums;           // the sums of weighted values, not divided, with what the weights refer to and their sum
    float* ml;
};
// For row r_tile of the piece; `first_lane` says (in a batch behind prefixes) where the row's parts are to be found.
static_assert(kSharesCap <= 1 << kRefPlace && kTileRows <= 1 << 10 && kRefPlace + 10 <= 24, "a reference is a share, a row of its tile and a bit");
template <class C>
__device__ __forceinline__ Target<C> target_of(const Args& a, const Piece& p, int r_tile, bool first_lane) {
    const Place at = place_of(a, p.q.row0, p.hk, p.rt * C::kM + r_tile);
    const size_t row = (size_t)at.row * a.H + at.head;
    const bool prefix = C::kOp == kShared && p.q.base == 1 << 30;
    const bool joined = C::kOp == kShared && (prefix || p.q.k_first > 0);  // two items make the row
    if (p.whole && !joined) {
        if (C::kOp == kShared && first_lane) {
            const size_t n = (size_t)a.N_cap * a.H;
            a.refs[2 * (n + row)] = -1;  // nothing is left to be joined
        }
        return Target<C>{(typename C::Out*)a.out + row * C::kDv, a.lse ? a.lse + row : nullptr, nullptr, nullptr};
    }
    if (C::kOp == kShared && first_lane && p.t0 == 0) {  // whoever begins the item says where its pieces are
        const size_t n = (size_t)a.N_cap * a.H, k = prefix ? row : n + row;
        a.refs[2 * k] = p.whole ? 0 : p.pieces;
        a.refs[2 * k + 1] = p.share0 | r_tile << kRefPlace | (p.q.k_first > 0 ? kRefPrefix : 0);
    }
    if (p.whole) {
        const size_t n = (size_t)a.N_cap * a.H, k = prefix ? row : n + row;
        return Target<C>{nullptr, nullptr, a.row_o + k * C::kDv, a.row_ml + k * 4};
    }
    const size_t k = (size_t)p.slot * a.m_cap + r_tile;
    return Target<C>{nullptr, nullptr, a.part_o + k * C::kDv, a.part_ml + k * 4};
}

// Result of a row's share of the keys: sums o[4] at columns d .. d + 3 (called for all of the lane's columns), what the weights refer to
// (-inf: no key), their sum l.
template <class C, class ForEach4>
__device__ __forceinline__ void hand_over(const Args& a, const Piece& p, int r_tile, bool first_lane, Reference of, float l, ForEach4 each) {
    const Target<C> to = target_of<C>(a, p, r_tile, first_lane);
    if (to.out) {
        const float inv = inverse(l);
        each([&](int d, f32x4 x) { store4(to.out + d, x * inv); });
        if (first_lane && to.lse) *to.lse = log_sum<C::kOp>(of, l, a.scale);
    } else {
        if constexpr (C::kOp == kTree) {  // as the lanes hold them: 64 lanes' four columns beside each other
            float* at = a.part_o + (size_t)p.slot * a.m_cap * C::kDv + (r_tile / C::kPartRows) * (C::kDv / C::kPartColumns) * 256 + (threadIdx.x & 63) * 4;
            const Buffer sums = buffer_at((const char*)a.part_o, 0x7fffffffu);
            const int base = (int)((at - a.part_o) * 4);
            each([&](int d, f32x4 x) { store_through(sums, base + (d / C::kPartColumns) * 1024, x); });
        } else {
            each([&](int d, f32x4 x) { store4(to.sums + d, x); });
        }
        if (first_lane) store4(to.ml, f32x4{of.raw, of.log2, l, 0.0f});
    }
}

// ---------------------------------------------------------------------------------------------------------------
// Products in fp32: every wave takes 16 rows of the tile, with operands straight from memory.  S^T = K Q^T and O^T = V^T P^T
// on v_mfma_f32_16x16x4_f32; the accumulator layout of S^T (lane: keys 4 (lane / 16) + e, row lane % 16) is the operand
// layout of P^T if step e of the second product takes keys 4 g + e of lane group g.
// Bound by latency where calls are short: 8 requests behind 437 common keys take 11 us and 5 to join; at 16 rows a wave every wave fetches
// its keys for itself, which the caches serve.
// ---------------------------------------------------------------------------------------------------------------
template <int OP, int KH, int KT, int DV>
struct Simple {
    static constexpr int kOp = OP, kHead = KH, kTail = KT, kDk = KH + KT, kDv = DV;
    static constexpr int kM = 64, kKeys = 32, kBlockThreads = kThreads, kPerUnit = 1;  // (kPerUnit: workgroups of a compute unit)
    static constexpr int kItemCost = 2;  // key tiles that taking up an item is worth (measured: 14000 cycles against 7000)
    static constexpr bool kEven = false; // (even pieces)
    static constexpr int kMinShare = 1;  // units of a share of a short line: a tile of its own costs less than waiting for a neighbour's
    static constexpr int kPartRows = 16, kPartColumns = 16;  // of a wave; for each four of a lane
    typedef float Out;
};

// Last key that packed row r sees (of a tree: that it may see).
template <int OP = kLatent>
__device__ __forceinline__ int last_key(const Args& a, const Seq& q, int r) {
    if constexpr (OP == kTree) return q.k_end - 1;
    return min(q.k_end - 1, q.base + (int)((uint32_t)r / (uint32_t)a.G));
}
// The last one up to which it sees them all.
template <int OP>
__device__ __forceinline__ int last_common_key(const Args& a, const Seq& q, int r) {
    if constexpr (OP == kTree) return q.base - 1;
    return last_key<OP>(a, q, r);
}

// Which of the 32 keys from `key` on a row of a tree sees, a bit each: the keys in front of `base` and what the row's bits say (bits that
// the mask does not hold are zero).
__device__ __forceinline__ uint32_t tree_window(const uint32_t* row, int words, int base, int key) {
    const int off = key - base;
    if (off <= -32) return 0xffffffffu;
    const int w = off >> 5, sh = off & 31;  // (off < 0: word -1 is all ones)
    const uint32_t lo = w < 0 ? 0xffffffffu : w < words ? row[w] : 0u, hi = w + 1 < words ? row[w + 1] : 0u;
    return (uint32_t)((((uint64_t)hi << 32) | lo) >> sh);
}

template <class C>
__device__ __forceinline__ void run_simple(const Args& a, const Piece& p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, li = lane & 15, lg = lane >> 4;
    const int n_packed = p.q.rows * a.G, first = p.rt * C::kM + wave * 16;
    if (first >= n_packed) return;
    const int r = min(first + li, n_packed - 1);
    const Place at = place_of(a, p.q.row0, p.hk, r);
    const float* qp = (const float*)a.q + ((size_t)at.row * a.H + at.head) * C::kDk;
    f32x4 q[C::kDk / 16];
#pragma unroll
    for (int s = 0; s < C::kDk / 16; ++s) q[s] = *reinterpret_cast<const f32x4*>(qp + 16 * s + 4 * lg);
    const int seen = last_key<C::kOp>(a, p.q, r);
    const uint32_t* tree = C::kOp == kTree ? a.tree + (size_t)at.row * a.tree_words : nullptr;
    f32x4 acc[C::kDv / 16];
#pragma unroll
    for (int b = 0; b < C::kDv / 16; ++b) acc[b] = f32x4{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f;
    const int k_first = p.q.k_begin + p.t0 * C::kKeys, k_last = min(p.q.k_begin + p.t1 * C::kKeys, p.q.k_end);
    // Where the next 16 keys lie is fetched while these are multiplied; where there are registers for it (not in the latent form) their
    // rows too, and these ones' values before their weights are known.
    constexpr int kSteps = C::kDk / 16, kBlocks = C::kDv / 16;
    constexpr bool kEarly = kSteps <= 12;
    auto slot_at = [&](int kb) { return slot_of<C::kOp>(a, find_key<C::kOp>(a, p.q, min(kb + li, k_last - 1))); };
    auto key_of = [&](uint32_t slot, int s) {
        const char* part = s < C::kHead / 16 ? a.k_head + (size_t)slot * a.head_stride + (size_t)p.hk * a.head_hk + 64 * s : a.k_tail + (size_t)slot * a.tail_stride + 64 * (s - C::kHead / 16);
        return *reinterpret_cast<const f32x4*>(part + 16 * lg);
    };
    auto value_of = [&](uint32_t slot, int e, int b) {
        const uint32_t vs = (uint32_t)__shfl((int)slot, 4 * lg + e, kWave);
        return ((const float*)(a.v + (size_t)vs * a.v_stride + (size_t)p.hk * a.v_hk))[16 * b + li];
    };
    uint32_t slot = k_first < k_last ? slot_at(k_first) : 0;
    f32x4 key[kEarly ? kSteps : 1];
    if (kEarly && k_first < k_last)
#pragma unroll
        for (int s = 0; s < kSteps; ++s) key[kEarly ? s : 0] = key_of(slot, s);
#pragma unroll 1
    for (int kb = k_first; kb < k_last; kb += 16) {
        const uint32_t now = slot;
        slot = slot_at(kb + 16);  // (behind the last key: that one's again)
        float value[kEarly ? 4 : 1][kBlocks];
        if constexpr (kEarly)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) value[e][b] = value_of(now, e, b);
        f32x4 z = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const f32x4 k4 = kEarly ? key[kEarly ? s : 0] : key_of(now, s);
#pragma unroll
            for (int e = 0; e < 4; ++e) z = __builtin_amdgcn_mfma_f32_16x16x4f32(k4[e], q[s][e], z, 0, 0, 0);
        }
        if constexpr (kEarly)
#pragma unroll
            for (int s = 0; s < kSteps; ++s) key[s] = key_of(slot, s);
        float top = -INFINITY;
        const uint32_t window = C::kOp == kTree ? tree_window(tree, a.tree_words, p.q.base, kb) : 0xffffffffu;
        auto sees_key = [&](int e) {
            const int key = kb + 4 * lg + e;
            return key >= p.q.k_first && key <= seen && key < k_last && (C::kOp != kTree || (window >> (4 * lg + e) & 1));
        };
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            z[e] = sees_key(e) ? z[e] : -INFINITY;
            top = fmaxf(top, z[e]);
        }
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        const float m_new = fmaxf(m, top);  // (of the products: their multiples by log2(e) may be beyond fp32)
        const float m_use = m_new == -INFINITY ? 0.0f : m_new;
        const float alpha = __builtin_amdgcn_exp2f((m - m_use) * a.scale_log2);
        f32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __builtin_amdgcn_exp2f((z[e] - m_use) * a.scale_log2);
        l = l * alpha + ((x[0] + x[1]) + (x[2] + x[3]));
        m = m_new;
#pragma unroll
        for (int b = 0; b < C::kDv / 16; ++b) acc[b] *= alpha;
        const bool masked = __any(kb + 15 > seen || kb + 15 >= k_last || kb < p.q.k_first || (C::kOp == kTree && (window & 0xffffu) != 0xffffu));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float v[kBlocks];
            uint32_t odd = 0;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                v[b] = kEarly ? value[kEarly ? e : 0][b] : value_of(now, e, b);
                odd |= (__builtin_bit_cast(uint32_t, v[b]) & 0x7f800000u) == 0x7f800000u;
            }
            const float sees = sees_key(e) ? 1.0f : 0.0f;
            if (!masked || !__any(odd)) {
#pragma unroll
                for (int b = 0; b < C::kDv / 16; ++b) acc[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[b], x[e], acc[b], 0, 0, 0);
            } else {
                // a value that is not finite must not meet the zero weight of a row that does not see it: each kind is
                // multiplied as 1 and takes its place in rows that see it, however small the weight
#pragma unroll
                for (int b = 0; b < C::kDv / 16; ++b) {
                    const bool fine = (__builtin_bit_cast(uint32_t, v[b]) & 0x7f800000u) != 0x7f800000u;
                    acc[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(fine ? v[b] : 0.0f, x[e], acc[b], 0, 0, 0);
                    const f32x4 none = {0, 0, 0, 0};
                    const f32x4 up = __builtin_amdgcn_mfma_f32_16x16x4f32(v[b] == INFINITY ? 1.0f : 0.0f, sees, none, 0, 0, 0);
                    const f32x4 down = __builtin_amdgcn_mfma_f32_16x16x4f32(v[b] == -INFINITY ? 1.0f : 0.0f, sees, none, 0, 0, 0);
                    const f32x4 nan = __builtin_amdgcn_mfma_f32_16x16x4f32(v[b] != v[b] ? 1.0f : 0.0f, sees, none, 0, 0, 0);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        float add = up[u] != 0.0f ? INFINITY : 0.0f;
                        add += down[u] != 0.0f ? -INFINITY : 0.0f;
                        acc[b][u] += nan[u] != 0.0f ? __builtin_nanf("") : add;
                    }
                }
            }
        }
    }
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    if (first + li < n_packed)
        hand_over<C>(a, p, wave * 16 + li, lg == 0, Reference{m, 0.0f}, l, [&](auto put) {
#pragma unroll
            for (int b = 0; b < C::kDv / 16; ++b) put(16 * b + 4 * lg, acc[b]);
        });
}

// ---------------------------------------------------------------------------------------------------------------
// bf16, heads of 64 and 128: a workgroup takes 128 rows, a wave 32 of them, and 64 keys at a time through LDS.
//
// S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_32x32x16_bf16.  A lane holds, of 32 keys, the scores of one row (row = lane % 32,
// keys 8 (e / 4) + 4 (lane / 32) + e % 4 for e < 16), so that statistics of a row take one exchange between the lane halves, and
// eight scores in a row are the operand of P^T for 16 keys, if V^T is read with its keys in the same order: two transposing LDS
// reads of four keys each.  The queries stay in registers, scores and weights never leave them.  K and V go from memory to LDS
// without passing through registers, the next tile while this one is computed.
//
// LDS rows are read across (16 bytes of each of 32 keys) and, for V^T, in blocks of 4 keys x 32 bytes; their 16-byte chunks are
// permuted by row such that both reach all banks.
// ---------------------------------------------------------------------------------------------------------------
//
// What bounds it: each of the four waves reads all keys and values of a tile, 128 KB with heads of 128 (160 KB with a second part of 64)
// and 32 KB (40) to write, 1280 (1600) cycles of a compute unit's LDS against 1024 (1280) of its matrix cores and 900 of exponentials
// and conversions.  Measured: 2048 rows of 32 heads behind 6000 tokens of context: 314-341 us by card, 938-864 TFLOP/s; a workgroup's 111
// tiles and two pieces take 496 000 cycles at 1.74 GHz (short calls run at 2.1-2.3), 4050 a tile, 2025 a tile of the unit, which two
// workgroups share.  (64 rows a wave would halve what LDS delivers, but leave one wave to a SIMD.)
//
// PAGES16: 16 keys from a multiple of 16 on are 16 rows that follow each other (no pages, or pages of a multiple of 16 tokens).
template <int OP, int KH, int KT, int DV, class OUT, bool PAGES16>
struct Tiled {
    static constexpr bool kPages16 = PAGES16;
    static constexpr int kOp = OP, kHead = KH, kTail = KT, kDk = KH + KT, kDv = DV;
    // Weights enter the second product as a pair of bf16 where results are fp32.  For bf16 results each is rounded once, by 2^-8 at most and to
    // either side, which is no more than the results' own rounding: 12 trees behind long contexts take 300 us, not 370.
    static constexpr bool kPair = sizeof(OUT) == 4;
    static constexpr int kM = kTileRows, kKeys = 64;
    static constexpr int kBlockThreads = kThreads, kWaves = row_tiles::kWaves;
    static constexpr int kPartRows = 32, kPartColumns = 8;  // of a wave; for each four of a lane
    static constexpr int kPerUnit = 2;                // workgroups of a compute unit, two waves to a SIMD
    static constexpr int kItemCost = OP == kTree ? 7 : 5;  // measured: 20000 cycles (loads that nothing hides, tiles with masked keys, sums on their way out) against 4000 a tile; of trees 23000 against 3100
    static constexpr int kMinShare = OP == kTree ? 1 : kItemCost + 1;  // (18 trees of 25-34 rows behind 221 tokens, 8/2 heads of 64: 15.6 us, not 19.7)
    static constexpr bool kEven = false;
    static constexpr int kHeadAt = 0, kTailAt = kKeys * KH * 2, kVAt = kTailAt + kKeys * KT * 2;
    static constexpr int kBuf = kVAt + kKeys * DV * 2;
    typedef OUT Out;
};

// Where chunk c of LDS row `row` with CH chunks of 16 bytes lies: at c ^ permutation.
template <int CH>
__device__ __forceinline__ int permutation(int row) { return CH >= 16 ? (row & 7) << 1 : CH == 8 ? row & 7 : (row >> 2) & 3; }

__device__ __forceinline__ void to_lds(const char* from, char* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// The same by a buffer descriptor, a lane's offset and a common one.  (Not only fewer instructions: behind a load in the other form the
// compiler takes every wait for an LDS read to be one for all of them.)
__device__ __forceinline__ void to_lds(Buffer from, int lane_at, int at, char* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, lane_at, at, 0, 0);
}

// A wave's part of 64 rows of CH chunks: load `i` of kEach takes rows (wave * kEach + i) * kRows ..; lane k of the wave holds the slot of row k.
template <int CH, int WAVES>
struct RowLoads {
    static constexpr int kRows = 64 / CH, kLoads = 64 / kRows, kEach = (kLoads + WAVES - 1) / WAVES;
    static __device__ __forceinline__ void issue(int i, const char* base, uint32_t stride, uint32_t slot, char* to, int wave, int lane) {
        if (kLoads % WAVES != 0 && wave * kEach + i >= kLoads) return;
        const int row0 = (wave * kEach + i) * kRows, row = row0 + lane / CH;
        const uint32_t at = kRows == 1 ? (uint32_t)__builtin_amdgcn_readlane((int)slot, row0) : (uint32_t)__shfl((int)slot, row, kWave);
        to_lds(base + (uint64_t)at * stride + (((lane % CH) ^ permutation<CH>(row)) << 4), to + row0 * CH * 16);
    }
};

// The tile's loads, which this wave has issued, have arrived, and so have everyone's behind the barrier; nobody reads what has been
// read in front of it any more.
__device__ __forceinline__ void arrive() {
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    __syncthreads();
}

// A barrier for what waves hand each other through LDS: loads that are on their way there stay so.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A wave's loads of a tile: of keys' first and second parts and of values, rows 16 wave .. 16 wave + 15 each.  Where they lie is fetched a
// tile ahead.  Of rows that follow each other every load has a descriptor and two offsets; else a lane holds the slot of a row.
template <class C>
struct TileLoads {
    static constexpr int CH = C::kHead / 8, CT = C::kTail / 8, CV = C::kDv / 8;
    typedef RowLoads<CH, C::kWaves> Head;
    typedef RowLoads<CT ? CT : 1, C::kWaves> Tail;
    typedef RowLoads<CV, C::kWaves> Value;
    static constexpr int kTails = CT ? Tail::kEach : 0, kEach = Head::kEach + kTails + Value::kEach;
    Where next;
    int next_key;        // the wave's first (of rows that follow each other)
    uint32_t slot;
    Buffer head, tail, value;
    int head_xor, head_add, tail_at, value_xor, value_add;

    __device__ __forceinline__ void place_lane(const Args& a, int lane) {
        head_xor = ((lane % CH) ^ permutation<CH>(lane / CH)) << 4;
        head_add = (lane / CH) * (int)a.head_stride;
        if constexpr (CT > 0) tail_at = (lane / CT) * (int)a.tail_stride + (((lane % CT) ^ permutation<CT>(lane / CT)) << 4);
        value_xor = ((lane % CV) ^ permutation<CV>(lane / CV)) << 4;
        value_add = (lane / CV) * (int)a.v_stride;
    }
    __device__ __forceinline__ void find(const Args& a, const Piece& p, int t, int wave, int lane) {
        const int key = p.q.k_begin + t * C::kKeys;
        next_key = C::kPages16 ? min(key + 16 * wave, (p.q.k_end - 1) & ~15) : min(key + lane, p.q.k_end - 1);
        next = find_key<C::kOp>(a, p.q, next_key);
    }
    // The loads to come are those of the tile that has been found.
    __device__ __forceinline__ void take(const Args& a, const Piece& p) {
        slot = slot_of<C::kOp>(a, next);
        if constexpr (C::kPages16) {
            slot = (uint32_t)uniform((int)slot);
            // (behind the last key there may be no row: a load from there is zeros)
            const uint32_t rows = C::kOp == kExpanded ? min((uint32_t)a.T_cap - min(slot, (uint32_t)a.T_cap), 16u) : 16u;
            // (A tree's values in a page's free slots, which may be anything and meet weights of 0, are zeros too.)
            const uint32_t values = C::kOp == kTree ? (uint32_t)min(p.q.k_end - next_key, 16) : rows;
            auto at = [&](const char* base, uint32_t stride, uint32_t n) { return buffer_at(base + (uint64_t)slot * stride, n ? (n - 1) * stride + stride : 0u); };
            head = at(a.k_head + (size_t)p.hk * a.head_hk, a.head_stride, rows);
            if constexpr (CT > 0) tail = at(a.k_tail, a.tail_stride, rows);
            value = at(a.v + (size_t)p.hk * a.v_hk, a.v_stride, values);
        }
    }
    // (Where rows may end inside the 16, in the expanded form and among a tree's values, all of the offset is the lane's: that is what is held
    // against the descriptor.)
    template <bool ENDS = C::kOp == kExpanded>
    static __device__ __forceinline__ void get(Buffer from, int lane_at, int at, char* to) {
        if constexpr (ENDS) to_lds(from, lane_at + at, 0, to);
        else to_lds(from, lane_at, at, to);
    }
    __device__ __forceinline__ void issue(int i, const Args& a, const Piece& p, char* buf, int wave, int lane) const {
        if (i < Head::kEach) {
            const int k = i * Head::kRows;
            if constexpr (C::kPages16) get(head, (head_xor ^ ((k & 7) << 5)) + head_add, k * (int)a.head_stride, buf + C::kHeadAt + (16 * wave + k) * C::kHead * 2);
            else Head::issue(i, a.k_head + (size_t)p.hk * a.head_hk, a.head_stride, slot, buf + C::kHeadAt, wave, lane);
        } else if (i < Head::kEach + kTails) {
            const int j = i - Head::kEach, k = j * Tail::kRows;
            if constexpr (C::kPages16) get(tail, tail_at, k * (int)a.tail_stride, buf + C::kTailAt + (16 * wave + k) * C::kTail * 2);
            else Tail::issue(j, a.k_tail, a.tail_stride, slot, buf + C::kTailAt, wave, lane);
        } else {
            const int j = i - Head::kEach - kTails, k = j * Value::kRows;
            if constexpr (C::kPages16) get<C::kOp == kExpanded || C::kOp == kTree>(value, (value_xor ^ ((k & 7) << 5)) + value_add, k * (int)a.v_stride, buf + C::kVAt + (16 * wave + k) * C::kDv * 2);
            else Value::issue(j, a.v + (size_t)p.hk * a.v_hk, a.v_stride, slot, buf + C::kVAt, wave, lane);
        }
    }
};

__device__ __forceinline__ float other_half(float x) {  // of the lane 32 further
    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    const uint32_t lo = both[0], hi = both[1];
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? lo : hi);
}

// Kinds of elements of an operand: the finite ones, or 1 where an element is of the kind.
enum : int { kFinite = 0, kUp = 1, kDown = 2, kNan = 3 };
__device__ __forceinline__ bf16x8 elements(s16x8 x, int kind) {
    s16x8 y;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t b = (uint16_t)x[k];
        const bool odd = (b & 0x7f80u) == 0x7f80u;
        const int is = !odd ? kFinite : b == 0x7f80u ? kUp : b == 0xff80u ? kDown : kNan;
        y[k] = (short)(is != kind ? 0u : odd ? 0x3f80u : b);
    }
    return __builtin_bit_cast(bf16x8, y);
}
__device__ __forceinline__ float odd_value(int kind) { return kind == kUp ? INFINITY : kind == kDown ? -INFINITY : __builtin_nanf(""); }
// Adds the value of the kind where it has weight.
__device__ __forceinline__ void put_odd(f32x16& acc, const f32x16& weight, int kind) {
    const float value = odd_value(kind);
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] += weight[e] != 0.0f ? value : 0.0f;
}

__device__ __forceinline__ f32x16 product(bf16x8 x, bf16x8 y, f32x16 sum) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, sum, 0, 0, 0); }
__device__ __forceinline__ f32x16 zeros() {
    f32x16 x;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = 0.0f;
    return x;
}
// N products in order: product(k, operand k), operands by read(k) AHEAD products before they are needed, and beside(k) in between.  (Left to
// itself the compiler saves registers and waits for every operand: 36 steps took 6000 cycles instead of 1300.)
template <int N, int AHEAD, class Operand, class Read, class Product, class Beside>
__device__ __forceinline__ void in_turn(Read read, Product product, Beside beside) {
    constexpr int A = N < AHEAD ? N : AHEAD;
    Operand x[A];
#pragma unroll
    for (int k = 0; k < A; ++k) x[k] = read(k);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        __builtin_amdgcn_sched_barrier(0);
        product(k, x[k % A]);
        if (k + A < N) x[k % A] = read(k + A);
        beside(k);
    }
    __builtin_amdgcn_sched_barrier(0);
}
// Sum of key(s) q[s] over N steps.
template <int N, class Key, class Beside>
__device__ __forceinline__ f32x16 first_product(Key key, const bf16x8* q, Beside beside) {
    f32x16 sum = zeros();
    in_turn<N, 8, bf16x8>(key, [&](int s, bf16x8 k) __attribute__((always_inline)) { sum = product(k, q[s], sum); }, beside);
    return sum;
}
// Eight keys of 32 columns, one column a lane: four keys at each of two places.
__device__ __forceinline__ s16x8 transposed(const char* four, const char* other_four) {
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)four), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)other_four);
    return s16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
}
__device__ __forceinline__ bool any_odd(s16x8 x) {  // an element that is not finite
    bool odd = false;
#pragma unroll
    for (int k = 0; k < 8; ++k) odd |= ((uint16_t)x[k] & 0x7f80u) == 0x7f80u;
    return odd;
}

template <class C>
struct Rows {
    static constexpr int kHeadSteps = C::kHead / 16, kTailSteps = C::kTail / 16, kBlocks = C::kDv / 32;
    // LDS offsets of a lane's operands repeat after 16 chunks (128 elements): the permutation changes the last four bits of a chunk's number
    static constexpr int kOwnK = std::min(kHeadSteps, 8), kOwnV = std::min(kBlocks, 4);
    bf16x8 q[kHeadSteps + kTailSteps];
    f32x16 acc[kBlocks];
    Reference of;        // of the row's weights
    float l;             // sum of this lane's weights
    int seen;            // last key of the lane's row
    const uint32_t* tree; // tree: the row's bits
    int tree_words, tree_base;
    int k_at[kOwnK], tail_at[std::max(kTailSteps, 1)], v_at[kOwnV];

    __device__ __forceinline__ void place_operands(int lane) {
        const int li = lane & 31, h = lane >> 5;
        constexpr int CH = C::kHead / 8, CT = C::kTail / 8, CV = C::kDv / 8;
#pragma unroll
        for (int s = 0; s < kOwnK; ++s) k_at[s] = li * CH * 16 + (((2 * s + h) ^ permutation<CH>(li)) << 4);
        if constexpr (CT > 0)
#pragma unroll
            for (int s = 0; s < kTailSteps; ++s) tail_at[s] = li * CT * 16 + (((2 * s + h) ^ permutation<CT>(li)) << 4);
        // lane g of 16 fetches 8 bytes of key row g / 4 of four, for 16 columns
        const int g = lane & 15, r = 4 * h + (g >> 2), column = lane & 16;
#pragma unroll
        for (int b = 0; b < kOwnV; ++b) v_at[b] = r * CV * 16 + (g & 1) * 8 + ((((32 * b + column) / 8 + ((g & 3) >> 1)) ^ permutation<CV>(r)) << 4);
    }
};

__device__ __forceinline__ float sum_of(const f32x16& z) {
    return (((z[0] + z[1]) + (z[2] + z[3])) + ((z[4] + z[5]) + (z[6] + z[7]))) + (((z[8] + z[9]) + (z[10] + z[11])) + ((z[12] + z[13]) + (z[14] + z[15])));
}
__device__ __forceinline__ float largest(const f32x16& z) {
    float top = fmaxf(z[0], z[1]);
#pragma unroll
    for (int e = 2; e < 16; ++e) top = fmaxf(top, z[e]);
    return fmaxf(top, other_half(top));
}
// Weights of the scores; their sum.  (Where nothing has been seen, the reference is -inf, and so are the scores.)
__device__ __forceinline__ float weights_of(f32x16& z, Reference of, float scale_log2) {
    const Reference use{of.raw, of.log2 == -INFINITY ? 0.0f : of.log2};
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = __builtin_amdgcn_exp2f(exponent(z[e], use, scale_log2));
    return sum_of(z);
}
// Eight weights as an operand.
__device__ __forceinline__ bf16x8 operand_of(const f32x16& z, int s) {
    return __builtin_bit_cast(bf16x8, u32x4{bf16_pair(z[8 * s], z[8 * s + 1]), bf16_pair(z[8 * s + 2], z[8 * s + 3]), bf16_pair(z[8 * s + 4], z[8 * s + 5]),
                                            bf16_pair(z[8 * s + 6], z[8 * s + 7])});
}

// Scores of 32 keys of the tile in `buf`; beside(s) is called between the products.
template <class C, class Beside>
__device__ __forceinline__ f32x16 scores_of(const Rows<C>& w, const char* buf, int block, Beside beside) {
    typedef Rows<C> R;
    const char *head = buf + C::kHeadAt + block * 32 * C::kHead * 2, *tail = buf + C::kTailAt + block * 32 * C::kTail * 2;
    return first_product<R::kHeadSteps + R::kTailSteps>([&](int s) __attribute__((always_inline)) {
        return *reinterpret_cast<const bf16x8*>(s < R::kHeadSteps ? head + w.k_at[s % R::kOwnK] + (s / R::kOwnK) * 256 : tail + w.tail_at[s < R::kHeadSteps ? 0 : s - R::kHeadSteps]);
    }, w.q, beside);
}
template <class C>
__device__ __forceinline__ s16x8 values_of(const Rows<C>& w, const char* buf, int block, int s, int b) {
    const char* at = buf + C::kVAt + (block * 32 + 16 * s) * C::kDv * 2 + w.v_at[b % Rows<C>::kOwnV] + (b / Rows<C>::kOwnV) * 256;
    return transposed(at, at + 8 * C::kDv * 2);
}

// Weights of 32 keys, two at a time, as operands (a pair of them where results are fp32) and their sum.
template <bool PAIR>
struct Weights {
    uint32_t hi[8], lo[PAIR ? 8 : 1];
    float sum = 0.0f;
    __device__ __forceinline__ void take(int k, const f32x16& z, float use, float scale_log2) {
        const float x = __builtin_amdgcn_exp2f(fmaf(z[2 * k], scale_log2, -use)), y = __builtin_amdgcn_exp2f(fmaf(z[2 * k + 1], scale_log2, -use));
        sum += x + y;
        hi[k] = bf16_pair(x, y);
        if constexpr (PAIR) lo[k] = bf16_pair(x - __builtin_bit_cast(float, hi[k] << 16), y - __builtin_bit_cast(float, hi[k] & 0xffff0000u));
    }
    // Those of step s of n.
    __device__ __forceinline__ void take_part(int s, int n, const f32x16& z, float use, float scale_log2) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k >= s * 8 / n && k < (s + 1) * 8 / n) take(k, z, use, scale_log2);
    }
    static __device__ __forceinline__ bf16x8 operand(const uint32_t* x, int s) { return __builtin_bit_cast(bf16x8, u32x4{x[4 * s], x[4 * s + 1], x[4 * s + 2], x[4 * s + 3]}); }
};
__device__ __forceinline__ float largest_of_lane(const f32x16& z) {
    float top = fmaxf(z[0], z[1]);
#pragma unroll
    for (int e = 2; e < 16; ++e) top = fmaxf(top, z[e]);
    return top;
}

// A tile of 64 keys that every row of the wave sees whole, by references in powers of two.  True: a score is ahead of its row's reference, and
// nothing has been added.
// The weights of a half are computed beside the products of the other: a product takes 32 cycles, in which eight instructions can be issued.
template <class C, class Beside>
__device__ __forceinline__ bool take_tile(Rows<C>& w, const char* buf, float scale_log2, Beside beside) {
    typedef Rows<C> R;
    typedef Weights<C::kPair> W;
    constexpr int kSteps = R::kHeadSteps + R::kTailSteps, kProducts = 2 * R::kBlocks;
    const float use = w.of.log2 == -INFINITY ? 0.0f : w.of.log2;
    W x0, x1;
    const f32x16 z0 = scores_of<C>(w, buf, 0, [&](int s) __attribute__((always_inline)) { beside(s); });
    float top = -INFINITY;
    const f32x16 z1 = scores_of<C>(w, buf, 1, [&](int s) __attribute__((always_inline)) {
        beside(kSteps + s);
        if (s == 0) top = largest_of_lane(z0);
        x0.take_part(s, kSteps, z0, use, scale_log2);
    });
    if (__any(fmaxf(top, largest_of_lane(z1)) * scale_log2 > w.of.log2)) return true;
    __builtin_amdgcn_s_setprio(1);  // the wave beside this one on the SIMD, at its scores or weights, gives way: 4 % of a long prompt's time
    auto add = [&](int block, const W& x, auto between) __attribute__((always_inline)) {
        in_turn<kProducts, 6, s16x8>([&](int k) __attribute__((always_inline)) { return values_of<C>(w, buf, block, k / R::kBlocks, k % R::kBlocks); },
                                     [&](int k, s16x8 v) __attribute__((always_inline)) {
                                         const int b = k % R::kBlocks, s = k / R::kBlocks;
                                         w.acc[b] = product(__builtin_bit_cast(bf16x8, v), W::operand(x.hi, s), w.acc[b]);
                                         if constexpr (C::kPair) w.acc[b] = product(__builtin_bit_cast(bf16x8, v), W::operand(x.lo, s), w.acc[b]);
                                     },
                                     between);
    };
    add(0, x0, [&](int k) __attribute__((always_inline)) { x1.take_part(k, kProducts, z1, use, scale_log2); });
    w.l += x0.sum + x1.sum;
    add(1, x1, [](int) {});
    __builtin_amdgcn_s_setprio(0);
    return false;
}

// 32 keys of any tile, from key0 on: some may be masked, references move if they have to.
template <class C>
__device__ __forceinline__ void take_any_keys(Rows<C>& w, const char* buf, int block, int key0, int k_first, float scale_log2, int lane) {
    typedef Rows<C> R;
    const int h = lane >> 5;
    f32x16 z = scores_of<C>(w, buf, block, [](int) {});
    const uint32_t window = C::kOp == kTree ? tree_window(w.tree, w.tree_words, w.tree_base, key0) : 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int at = 8 * (e >> 2) + 4 * h + (e & 3), key = key0 + at;
        z[e] = key >= k_first && key <= w.seen && (C::kOp != kTree || (window >> at & 1)) ? z[e] : -INFINITY;
    }
    const float top = largest(z);
    // The reference keeps a distance above the largest score and is moved only when a score overtakes it: weights stay below one,
    // lose nothing (they are floating-point numbers) and the accumulators are rescaled a few times per row, not per tile.
    const bool ahead = exponent(top, w.of, scale_log2) > 0.0f;
    if (__any(ahead)) {
        const Reference old = w.of;
        if (ahead) w.of = reference_for(top, scale_log2);
        const float alpha = !ahead || old.log2 == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(distance(old, w.of, scale_log2));
        w.l *= alpha;
#pragma unroll
        for (int b = 0; b < R::kBlocks; ++b) w.acc[b] *= alpha;
    }
    w.l += weights_of(z, w.of, scale_log2);
    bf16x8 hi[2], lo[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) hi[s] = operand_of(z, s);
    if constexpr (C::kPair) {
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] -= (float)(__bf16)z[e];
#pragma unroll
        for (int s = 0; s < 2; ++s) lo[s] = operand_of(z, s);
    }
#pragma unroll
    for (int b = 0; b < R::kBlocks; ++b) {
        const s16x8 v0 = values_of<C>(w, buf, block, 0, b), v1 = values_of<C>(w, buf, block, 1, b);
        if (__any(any_odd(v0) | any_odd(v1))) {
            // a value that is not finite must not meet the zero weight of a row that does not see it: each kind is
            // multiplied as 1 and takes its place in rows that see it, however small the weight
            w.acc[b] = product(elements(v1, kFinite), hi[1], product(elements(v0, kFinite), hi[0], w.acc[b]));
            if constexpr (C::kPair) w.acc[b] = product(elements(v1, kFinite), lo[1], product(elements(v0, kFinite), lo[0], w.acc[b]));
#pragma unroll 1
            for (int kind = kUp; kind <= kNan; ++kind) {
                int first_key = key0 + 4 * h;
                asm volatile("" : "+v"(first_key));  // (computed for each kind and block: otherwise it is kept beside everything else)
                auto sees = [&](int s) {
                    u32x4 one;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int key = first_key + 16 * s + 8 * (k >> 1) + 2 * (k & 1);
                        const uint32_t bits = C::kOp == kTree ? window >> (key - key0) : 3u;
                        one[k] = (key >= k_first && key <= w.seen && (bits & 1) ? 0x3f80u : 0u) | (key + 1 >= k_first && key + 1 <= w.seen && (bits & 2) ? 0x3f800000u : 0u);
                    }
                    return __builtin_bit_cast(bf16x8, one);
                };
                put_odd(w.acc[b], product(elements(v1, kind), sees(1), product(elements(v0, kind), sees(0), zeros())), kind);
            }
        } else {
            w.acc[b] = product(__builtin_bit_cast(bf16x8, v1), hi[1], product(__builtin_bit_cast(bf16x8, v0), hi[0], w.acc[b]));
            if constexpr (C::kPair) w.acc[b] = product(__builtin_bit_cast(bf16x8, v1), lo[1], product(__builtin_bit_cast(bf16x8, v0), lo[0], w.acc[b]));
        }
    }
}

// False: with weights in pairs, an infinite value that has met the rest of a weight, of either sign or zero, is NaN (to look at the values in the
// loop over whole tiles would cost a third of it).  Sums that are not finite are not handed over; the piece is to be taken again without that loop.
template <class C>
__device__ __forceinline__ bool run_tiled(const Args& a, const Piece& p, char* buf0, char* buf1, bool fast) {
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), li = lane & 31, h = lane >> 5;
    const int n_packed = p.q.rows * a.G, first = p.rt * C::kM + wave * 32;
    const bool active = first < n_packed;  // a wave without rows helps to load
    typedef Rows<C> R;
    R w;
    w.of = Reference{0.0f, -INFINITY};
    w.l = 0.0f;
    w.seen = -1;
    w.place_operands(lane);
#pragma unroll
    for (int b = 0; b < R::kBlocks; ++b) w.acc[b] = zeros();
    int seen_first = 0, seen_last = 0;  // by the wave's first and last row
    if (active) {
        const int r = min(first + li, n_packed - 1);
        const Place at = place_of(a, p.q.row0, p.hk, r);
        const uint16_t* qp = (const uint16_t*)a.q + ((size_t)at.row * a.H + at.head) * C::kDk;
#pragma unroll
        for (int s = 0; s < C::kDk / 16; ++s) w.q[s] = *reinterpret_cast<const bf16x8*>(qp + 16 * s + 8 * h);
        w.seen = last_key<C::kOp>(a, p.q, r);
        if constexpr (C::kOp == kTree) {
            w.tree = a.tree + (size_t)at.row * a.tree_words;
            w.tree_words = a.tree_words;
            w.tree_base = p.q.base;
        }
        seen_first = last_common_key<C::kOp>(a, p.q, first);
        seen_last = last_key<C::kOp>(a, p.q, min(first + 31, n_packed - 1));
    }
    TileLoads<C> loads;
    loads.place_lane(a, lane);
    int t = p.t0;
    auto load_all = [&](char* to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < TileLoads<C>::kEach; ++i) loads.issue(i, a, p, to, wave, lane);
    };
    __syncthreads();  // nobody reads the buffers any more
    if (t < p.t1) {
        loads.find(a, p, t, wave, lane);
        loads.take(a, p);
        load_all(buf0);
        loads.find(a, p, min(t + 1, p.t1 - 1), wave, lane);
        auto whole = [&] { return active && t < p.t1 && p.q.k_begin + t * C::kKeys >= p.q.k_first && p.q.k_begin + t * C::kKeys + C::kKeys - 1 <= seen_first; };
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
            // the first tile, tiles with masked keys, tiles where a reference moves; every wave goes its own way, one barrier to a tile
            const bool odd = (t - p.t0) & 1;
            if (!loaded) {
                arrive();
                loads.take(a, p);
                loads.find(a, p, min(t + 2, p.t1 - 1), wave, lane);
                load_all(odd ? buf0 : buf1);
            }
            loaded = false;
            const int key0 = p.q.k_begin + t * C::kKeys;
            if (active)
#pragma unroll 1
                for (int block = 0; block < 2; ++block)
                    if (key0 + 32 * block <= seen_last) take_any_keys<C>(w, odd ? buf1 : buf0, block, key0 + 32 * block, p.q.k_first, a.scale_log2, lane);
            ++t;
            // all the others: here the sums are the products' alone (where something else may touch them, the compiler makes a second
            // set and copies them in every tile)
            // (Said to be one value for the wave: otherwise the loop saves masks around itself, 13 moves a tile, 2 % of a long prompt.)
            const bool near = uniform((int)__any(w.of.raw != 0.0f)) == 0;
            if (!odd && near && fast) {
                w.of.raw = 0.0f;  // (known, and in no register of the loop)
                while (whole()) {
                    if (!step(buf1, buf0)) { loaded = true; break; }
                    if (!whole()) break;
                    if (!step(buf0, buf1)) { loaded = true; break; }
                }
            }
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);  // the load too many has its place until it has come
    }
    if constexpr (C::kPair) {
        if (fast && p.t1 - p.t0 > 1) {
            float odd = 0.0f;
#pragma unroll
            for (int b = 0; b < R::kBlocks; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) odd = fmaf(w.acc[b][e], 0.0f, odd);
            __syncthreads();  // (all loads have come, nobody reads the buffers any more)
            int* any = reinterpret_cast<int*>(buf0);
            const int mine = __any(odd != 0.0f);
            if (lane == 0) any[wave] = mine;
            __syncthreads();
            if (uniform(any[0] | any[1] | any[2] | any[3])) return false;
        }
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

// How a workgroup takes a piece (trees: tree_tiles.hpp).
template <class C>
struct Pieces {
    static constexpr int kShared = 0;  // bytes of LDS besides the buffers
    static __device__ __forceinline__ bool take(const Args& a, const Piece& p, char* buf0, char* buf1, int*, bool fast) { return run_tiled<C>(a, p, buf0, buf1, fast); }
};

// The pieces of a share of the line, one after the other.
template <class C>
struct Walk {
    Line line;
    Seq q;
    long long seq_start, head_units;
    int s, hk, rt, tiles;
    bool inside;  // q is sequence s

    __device__ __forceinline__ void begin(const Args& a, int share, const Line& l) {
        line = l;
        s = l.seq;
        seq_start = l.seq_start;
        inside = false;
        if (C::kOp != kShared && threadIdx.x == 0) a.desc[(size_t)share * kDescInts] = 0;
    }
    __device__ __forceinline__ bool next(const Args& a, int share, Piece& p) {
        const int n = n_sequences<C::kOp>(a);
        for (;;) {
            if (!inside) {
                if (s >= n || seq_start >= line.hi) return false;
                q = line.known && s == line.seq ? line.first : sequence<C::kOp>(a, s);
                tiles = row_tiles_of<C>(a, q);
                head_units = units_before<C>(a, q, tiles);
                hk = rt = 0;
                if (tiles == 0) {
                    ++s;
                    continue;
                }
                if (seq_start < line.lo) {  // the stream head and the row tile that hold unit lo
                    hk = (int)quotient(line.lo - seq_start, head_units);
                    const long long head_start = seq_start + hk * head_units;
                    int last = tiles - 1;
                    while (rt < last) {
                        const int mid = (rt + last + 1) >> 1;
                        if (head_start + units_before<C>(a, q, mid) <= line.lo) rt = mid; else last = mid - 1;
                    }
                }
                inside = true;
            }
            if (rt == tiles) {
                rt = 0;
                ++hk;
            }
            if (hk == a.H_stream) {
                seq_start += head_units * a.H_stream;
                ++s;
                inside = false;
                continue;
            }
            const long long item = seq_start + hk * head_units + units_before<C>(a, q, rt);
            if (item >= line.hi) return false;
            p.q = q;
            p.hk = hk;
            p.rt = rt++;
            const int nk = key_tiles<C>(a, q, p.rt);
            const long long t0 = line.lo - item - C::kItemCost, t1 = line.hi - item - C::kItemCost;
            p.t0 = t0 > 0 ? (int)min(t0, (long long)nk) : 0;
            p.t1 = t1 > 0 ? (int)min(t1, (long long)nk) : 0;
            if (nk == 0 ? item < line.lo : p.t0 >= p.t1) continue;  // nothing of it is this share's
            p.whole = p.t0 == 0 && p.t1 == nk;
            p.slot = 0;
            p.share0 = share;
            p.pieces = 1;
            if (!p.whole) {
                if constexpr (C::kOp != kTree) p.share0 = line.share_of(item + C::kItemCost);
                if (C::kOp != kTree || p.t0 == 0) p.pieces = line.share_of(item + C::kItemCost + nk - 1) - p.share0 + 1;  // (of a tree's item only the first needs to know)
                p.slot = 2 * share + (p.t0 == 0 ? 1 : 0);  // an item that begins here, or one that began before
                if (C::kOp != kShared && p.t0 == 0 && threadIdx.x == 0) {
                    int32_t* desc = a.desc + (size_t)share * kDescInts;
                    desc[1] = q.row0; desc[2] = hk; desc[3] = p.rt; desc[4] = min(q.rows * a.G - p.rt * C::kM, C::kM);
                    desc[5] = p.slot; desc[6] = p.slot + 1; desc[7] = 2;  // the first piece's slot, the second's, and from there on
                    desc[0] = p.pieces;
                }
            }
            return true;
        }
    }
};

// Neighbouring shares read the same keys: they go to the same one of the 8 dies (workgroups are dealt to them in turn).
__device__ __forceinline__ int share_of_block(int block, int nb) {
    const int per = nb >> 3, rest = nb & 7, die = block & 7;
    return (block >> 3) + die * per + min(die, rest);
}

template <class C>
__global__ __launch_bounds__(C::kBlockThreads, 1) void simple_kernel(Args a) {
    __shared__ long long scratch[kThreads + kWaves];
    const int share = share_of_block(blockIdx.x, a.nb);
    const Line line = C::kOp == kTree && a.B <= kWave ? find_share_by_wave<C>(a, share) : find_share<C>(a, share, scratch);
    Walk<C> walk;
    walk.begin(a, share, line);
    Piece p;
    while (walk.next(a, share, p)) run_simple<C>(a, p);
}

template <class C>
__global__ __launch_bounds__(C::kBlockThreads, 2) void tiled_kernel(Args a) {  // (256 registers: two waves on a SIMD)
    __shared__ __align__(1024) char buf0[C::kBuf];
    __shared__ __align__(1024) char buf1[C::kBuf];
    const int share = share_of_block(blockIdx.x, a.nb);
    const Line line = C::kOp == kTree && a.B <= kWave ? find_share_by_wave<C>(a, share) : find_share<C>(a, share, reinterpret_cast<long long*>(buf0));
    Walk<C> walk;
    walk.begin(a, share, line);
    Piece p;
    while (walk.next(a, share, p)) {
        bool fast = true;
        if constexpr (Pieces<C>::kShared > 0) {
            __shared__ int more[Pieces<C>::kShared / sizeof(int)];
            while (!Pieces<C>::take(a, p, buf0, buf1, more, fast)) fast = false;
        } else {
            while (!Pieces<C>::take(a, p, buf0, buf1, nullptr, fast)) fast = false;
        }
    }
}

template <class C>
struct Kernel;
template <int OP, int KH, int KT, int DV>
struct Kernel<Simple<OP, KH, KT, DV>> {
    static constexpr auto run = simple_kernel<Simple<OP, KH, KT, DV>>;
};
template <int OP, int KH, int KT, int DV, class OUT, bool PAGES16>
struct Kernel<Tiled<OP, KH, KT, DV, OUT, PAGES16>> {
    static constexpr auto run = tiled_kernel<Tiled<OP, KH, KT, DV, OUT, PAGES16>>;
};

// The reference of the piece, of a wave's 64, that is furthest ahead, and of `more`.
__device__ __forceinline__ Reference furthest(Reference x, Reference more, float scale_log2) {
    if (distance(more, x, scale_log2) > 0.0f) x = more;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const Reference y{__shfl_xor(x.raw, o, kWave), __shfl_xor(x.log2, o, kWave)};
        if (distance(y, x, scale_log2) > 0.0f) x = y;
    }
    return Reference{__shfl(x.raw, 0, kWave), __shfl(x.log2, 0, kWave)};  // (lanes may hold different ones of the same height)
}

// A row's result out of the sums of its `pieces`: a wave per row.  source(k) says where piece k has its sums and its (reference, sum of weights).
// The statistics of 64 pieces are fetched at once, a piece a lane, and then the sums one behind the other without waiting.
struct Source {
    const float* sums;
    const float* ml;
};
template <class C, class SourceOf>
__device__ __forceinline__ void join(const Args& a, int pieces, SourceOf source, typename C::Out* out, float* lse, int lane) {
    constexpr int kColumns = C::kDv / 64, kVector = kColumns < 4 ? kColumns : 4, kVectors = kColumns / kVector;
    constexpr Reference kNone{-INFINITY, 0.0f};
    float o[kColumns], l = 0.0f;
    Reference of = kNone;
#pragma unroll
    for (int c = 0; c < kColumns; ++c) o[c] = 0.0f;
    for (int first = 0; first < pieces; first += kWave) {
        const int n = min(pieces - first, kWave);
        const Source mine = source(first + min(lane, n - 1));
        const f32x4 stats = *reinterpret_cast<const f32x4*>(mine.ml);
        const float pl = lane < n ? stats[2] : 0.0f;
        const Reference pm = pl == 0.0f ? kNone : Reference{stats[0], stats[1]};  // (none: a piece without a visible key)
        // Any number near the furthest reference will do; where powers of two are too coarse for one, it is that reference itself.
        const float top = fmaxf(wave_max(fmaf(pm.raw, a.scale_log2, pm.log2)), fmaf(of.raw, a.scale_log2, of.log2));
        Reference use{0.0f, top};
        if (!(fabsf(top) <= kNear)) use = furthest(pm, of, a.scale_log2);
        const float before = l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(distance(of, use, a.scale_log2));
        const float w = pl == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(distance(pm, use, a.scale_log2));
        float sum = w * pl;
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x, kWave);
        l = l * before + sum;
        of = l == 0.0f ? kNone : use;
#pragma unroll
        for (int c = 0; c < kColumns; ++c) o[c] *= before;
        const uint32_t lo = (uint32_t)(uintptr_t)mine.sums, hi = (uint32_t)((uintptr_t)mine.sums >> 32);
        // The sums of `many` pieces at once.  (Left to itself the compiler fetches one piece, waits and fetches the next.  8000 keys, 128 heads,
        // 126 pieces: 91 us, not 42; eight at once where there are three, the last one again and again, cost a long prompt 30 us, not 20.)
        auto add = [&](int k0, auto many) __attribute__((always_inline)) {
            float y[many.value][kColumns];
#pragma unroll
            for (int i = 0; i < many.value; ++i) {
                const uintptr_t at = ((uintptr_t)(uint32_t)__builtin_amdgcn_readlane((int)hi, k0 + i) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)lo, k0 + i);
                typedef const __attribute__((address_space(1))) char global_char;
                global_char* x = (global_char*)at;
#pragma unroll
                for (int v = 0; v < kVectors; ++v) __builtin_memcpy(y[i] + v * kVector, x + (v * 64 * kVector + lane * kVector) * 4, kVector * 4);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < many.value; ++i) {
                const float wk = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), k0 + i));
#pragma unroll
                for (int c = 0; c < kColumns; ++c) o[c] = fmaf(wk, y[i][c], o[c]);
            }
        };
        int k = 0;
#pragma unroll 1
        for (; n - k >= 8; k += 8) add(k, std::integral_constant<int, 8>());
        if (n - k >= 4) add(k, std::integral_constant<int, 4>()), k += 4;
        if (n - k >= 2) add(k, std::integral_constant<int, 2>()), k += 2;
        if (n - k >= 1) add(k, std::integral_constant<int, 1>());
    }
    const float inv = inverse(l);
#pragma unroll
    for (int v = 0; v < kVectors; ++v) {
        typename C::Out y[kVector];
#pragma unroll
        for (int c = 0; c < kVector; ++c) {
            if constexpr (sizeof(typename C::Out) == 2) y[c] = (uint16_t)bf16_bits(o[v * kVector + c] * inv);
            else y[c] = o[v * kVector + c] * inv;
        }
        __builtin_memcpy(out + v * 64 * kVector + lane * kVector, y, sizeof y);
    }
    if (lse && lane == 0) *lse = log_sum<C::kOp>(of, l, a.scale);
}

// Joins the item of which a share has the first piece and others have more.  blockIdx.x: share, blockIdx.y: rows of the tile, kWaves at a time.
template <class C>
__global__ __launch_bounds__(kThreads) void join_shares_kernel(Args a) {
    const int32_t* desc = a.desc + (size_t)blockIdx.x * kDescInts;
    const int pieces = desc[0];
    if (pieces <= 0) return;
    const int lane = threadIdx.x & 63, first = desc[5], second = desc[6], step = desc[7];
    for (int r = blockIdx.y * kWaves + uniform(threadIdx.x >> 6); r < desc[4]; r += gridDim.y * kWaves) {
        const Place to = place_of(a, desc[1], desc[2], desc[3] * C::kM + r);
        const size_t row = (size_t)to.row * a.H + to.head;
        join<C>(a, pieces, [&](int k) {
            const size_t at = (size_t)(k == 0 ? first : second + (k - 1) * step) * a.m_cap + r;
            return Source{a.part_o + at * C::kDv, a.part_ml + at * 4};
        }, (typename C::Out*)a.out + row * C::kDv, a.lse ? a.lse + row : nullptr, lane);
    }
}

// Joins what a row's prefix and its own keys left.  A wave per (call row, query head), from `first` on.
template <class C>
__global__ __launch_bounds__(kThreads) void join_rows_kernel(Args a, size_t first) {
    const int lane = threadIdx.x & 63;
    const size_t n = (size_t)a.N_cap * a.H;
    const size_t row = first + (size_t)blockIdx.x * kWaves + uniform(threadIdx.x >> 6);
    if (row >= n) return;
    const int i0 = clamp_to(a.cu_groups[0], 0, a.B), i1 = clamp_to(a.cu_groups[a.n_groups], 0, a.B);
    const int call_row = (int)(row / a.H), head = (int)(row - (size_t)call_row * a.H);
    // (The references are read beside the bounds: what stands there for a row outside of them is not used.)
    const u32x2 own = reinterpret_cast<const u32x2*>(a.refs)[n + row], common = reinterpret_cast<const u32x2*>(a.refs)[row];
    if (call_row < a.cu_q[i0] || call_row >= a.cu_q[i1] || (int)own[0] < 0) return;  // (no prefix, and whole: written already)
    const bool behind = own[1] & kRefPrefix;
    const int pieces[2] = {behind ? clamp_to((int)common[0], 0, a.shares_cap) : -1, clamp_to((int)own[0], 0, a.shares_cap)};
    const int share0[2] = {(int)(common[1] & ((1 << kRefPlace) - 1)), (int)(own[1] & ((1 << kRefPlace) - 1))};
    const int place[2] = {min((int)(common[1] >> kRefPlace & 1023), a.m_cap - 1), min((int)(own[1] >> kRefPlace & 1023), a.m_cap - 1)};
    const int n0 = pieces[0] < 0 ? 0 : max(pieces[0], 1), n1 = max(pieces[1], 1);  // (no pieces: the whole in row_o)
    join<C>(a, n0 + n1, [&](int k) {
        const int part = k < n0 ? 0 : 1, j = part ? k - n0 : k;
        if (pieces[part] <= 0) return Source{a.row_o + (part * n + row) * C::kDv, a.row_ml + (part * n + row) * 4};
        const int share = clamp_to(share0[part] + j, 0, a.shares_cap - 1);
        const size_t at = (size_t)(2 * share + (j == 0 ? 1 : 0)) * a.m_cap + place[part];
        return Source{a.part_o + at * C::kDv, a.part_ml + at * 4};
    }, (typename C::Out*)a.out + row * C::kDv, a.lse ? a.lse + row : nullptr, lane);
}

// ---------------------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------------------
struct Layout {
    size_t part_o, part_ml, desc, row_o, row_ml, refs, total;
};

// Workspace: slots of two pieces per share, and for a batch behind shared prefixes two results per row and head.
inline Layout layout_of(int m_cap, int dv, long long rows, bool shared) {
    Layout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t p = at; at += align_up(bytes, 256); return p; };
    l.part_o = take((size_t)2 * kSharesCap * m_cap * dv * sizeof(float));
    l.part_ml = take((size_t)2 * kSharesCap * m_cap * 4 * sizeof(float));
    l.desc = take((size_t)2 * kSharesCap * kDescInts * sizeof(int32_t));
    if (shared) {
        l.row_o = take((size_t)2 * rows * dv * sizeof(float));
        l.row_ml = take((size_t)2 * rows * 4 * sizeof(float));
        l.refs = take((size_t)2 * rows * 2 * sizeof(int32_t));
    }
    l.total = at;
    return l;
}

inline void place(Args& a, const Layout& l, void* workspace) {
    char* w = (char*)workspace;
    a.part_o = (float*)(w + l.part_o);
    a.part_ml = (float*)(w + l.part_ml);
    a.desc = (int32_t*)(w + l.desc);
    a.row_o = (float*)(w + l.row_o);
    a.row_ml = (float*)(w + l.row_ml);
    a.refs = (int32_t*)(w + l.refs);
    a.shares_cap = kSharesCap;
}

// Compute units of the current device.
inline int compute_units() {
    static thread_local int cached_dev = -1, cached = 0;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) {
        (void)hipGetLastError();
        return 256;
    }
    if (dev != cached_dev) {
        int n = 0;
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) {
            (void)hipGetLastError();
            n = 256;
        }
        cached_dev = dev;
        cached = n;
    }
    return cached;
}

template <class C>
void launch_tree_join(const Args& a, hipStream_t s);  // (tree_tiles.hpp)

template <class C>
int launch(Args a, int max_workgroups, void* stream, const char* who) {
    int units = compute_units();
    if (max_workgroups > 0) units = std::min(units, max_workgroups);  // (any number is allowed: taken times the workgroups of a unit only now)
    a.nb = std::min(units * C::kPerUnit, kSharesCap);
    a.min_share = C::kMinShare;
    a.even_cap = a.nb;
    // Items that may outnumber the workgroups are cut into pieces for several rounds.  (Else that many descriptors need not be looked at.)
    if (C::kEven && kEvenRounds * a.nb <= 2 * kSharesCap && ((long long)a.N_cap * a.G + C::kM - 1) / C::kM + a.B > a.nb) a.even_cap = kEvenRounds * a.nb;
    hipStream_t s = (hipStream_t)stream;
    hipLaunchKernelGGL((Kernel<C>::run), dim3(a.nb), dim3(C::kBlockThreads), 0, s, a);
    int rc = check_launch(who);
    if (rc != FSR_OK) return rc;
    if constexpr (C::kOp == kShared) {  // (each operator's join is compiled for it alone)
        constexpr size_t kMost = (size_t)kMaxBlocks * kWaves;
        const size_t rows = (size_t)a.N_cap * a.H;
        for (size_t first = 0; first < rows; first += kMost) {
            const size_t now = std::min(rows - first, kMost);
            hipLaunchKernelGGL((join_rows_kernel<C>), dim3((unsigned)((now + kWaves - 1) / kWaves)), dim3(kThreads), 0, s, a, first);
        }
    } else if constexpr (C::kOp == kTree) {
        launch_tree_join<C>(a, s);
    } else {
        // 16 workgroups a share: one row a wave of a latent tile, two of a tile of heads; with 32 there the launching of workgroups took longer: 20 us, not 17.6
        hipLaunchKernelGGL((join_shares_kernel<C>), dim3(a.even_cap, std::min(16, (a.m_cap + kWaves - 1) / kWaves)), dim3(kThreads), 0, s, a);
    }
    return check_launch(who);
}

}  // namespace row_tiles
}  // namespace fsr
