// Cache append with the position rotation on the way: a call's query and key rows are turned to their positions, keys and values enter
// the request's pages.
//     first R elements of a head, pairs (a, b) = (x[i], x[i + R/2]) or (x[2i], x[2i + 1]):   a cos - b sin,  b cos + a sin
// Memory-bound: every element is read once and written once.  A workgroup takes a row; a thread takes 16 elements that are rotated with
// each other, or 8 that are only moved.  Its loads go out before the row's request, page and position are known (four round trips to
// memory one after the other: offsets, length and table, cosines).
#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "common.hpp"
#include "device_utils.hpp"

namespace fsr {
namespace {

constexpr int kThreads = 256, kAtOnce = 2;  // pieces of a thread that are loaded before the first is stored
constexpr int kMaxRows = 1 << 22;           // workgroups of a launch

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

struct RopeArgs {
    const void* q;
    const void* k_new;
    const void* v_new;
    const float* cos_sin;
    const int32_t* positions;
    const uint64_t* tree;
    void* q_out;
    void* k_cache;
    void* v_cache;
    const float* k_scale;
    const float* v_scale;
    const int32_t* bt;
    const int32_t* ctx;
    const int32_t* cu_q;
    long long q_stride, k_stride, v_stride;  // elements from a row to the next
    int B, N_cap, H_q, H_kv, D, R, P, max_pages, n_pages, T, tree_words, token_major;
    int turned, per_head, q_pieces, pieces;  // pieces of a head that are rotated, of a head, of the queries, of a row
};

// Eight elements.
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {
    u32x4 x;
    __device__ __forceinline__ void load(const uint16_t* p) { x = *reinterpret_cast<const u32x4*>(p); }
    __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<u32x4*>(p) = x; }
    __device__ __forceinline__ float get(int k) const {
        const uint32_t w = x[k >> 1];
        return __builtin_bit_cast(float, k & 1 ? w & 0xffff0000u : w << 16);
    }
    __device__ __forceinline__ void set(const float* v) {  // (rounded once, to nearest)
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            w[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector((__attribute__((ext_vector_type(2))) float){v[2 * k], v[2 * k + 1]}, __attribute__((ext_vector_type(2))) __bf16));
        x = u32x4{w[0], w[1], w[2], w[3]};
    }
};
template <>
struct Eight<float> {
    f32x4 x, y;
    __device__ __forceinline__ void load(const float* p) { x = *reinterpret_cast<const f32x4*>(p); y = *reinterpret_cast<const f32x4*>(p + 4); }
    __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<f32x4*>(p) = x; *reinterpret_cast<f32x4*>(p + 4) = y; }
    __device__ __forceinline__ float get(int k) const { return k < 4 ? x[k] : y[k - 4]; }
    __device__ __forceinline__ void set(const float* v) { x = f32x4{v[0], v[1], v[2], v[3]}; y = f32x4{v[4], v[5], v[6], v[7]}; }
};

// Where a piece of a row lies: its head (queries, keys, values one behind the other) and its elements.
struct At {
    int part, head, first, second;  // part 0 query, 1 key, 2 value; second < 0: eight elements that are moved as they are
    int turn;                       // the first of its eight angles
};
template <bool PAIRS>
__device__ __forceinline__ At piece_at(const RopeArgs& a, int n) {
    At p;
    const bool is_q = n < a.q_pieces;
    if (!is_q) n -= a.q_pieces;
    const int k_pieces = a.H_kv * a.per_head;
    if (!is_q && n >= k_pieces) {
        n -= k_pieces;
        const int each = a.D >> 3;
        p.part = 2;
        p.head = (int)((uint32_t)n / (uint32_t)each);
        p.first = (n - p.head * each) * 8;
        p.second = -1;
        return p;
    }
    p.part = is_q ? 0 : 1;
    p.head = (int)((uint32_t)n / (uint32_t)a.per_head);
    const int u = n - p.head * a.per_head;
    p.turn = 8 * u;
    if (u < a.turned) {
        p.first = PAIRS ? 16 * u : 8 * u;
        p.second = PAIRS ? 16 * u + 8 : 8 * u + a.R / 2;
    } else {
        p.first = a.R + 8 * (u - a.turned);
        p.second = -1;
    }
    return p;
}

template <typename T, bool PAIRS, bool KV8>
__global__ __launch_bounds__(kThreads) void rope_append_kernel(RopeArgs a) {
    for (int row = blockIdx.x; row < a.N_cap; row += gridDim.x) {
        const T* from[3] = {(const T*)a.q + row * a.q_stride, (const T*)a.k_new + row * a.k_stride, (const T*)a.v_new + row * a.v_stride};
        Eight<T> x[kAtOnce], y[kAtOnce];
        At at[kAtOnce];
        auto fetch = [&](int n, int s) __attribute__((always_inline)) {
            at[s] = piece_at<PAIRS>(a, min(n, a.pieces - 1));
            const T* p = (at[s].part == 0 ? from[0] : at[s].part == 1 ? from[1] : from[2]) + at[s].head * a.D;
            x[s].load(p + at[s].first);
            y[s].load(p + max(at[s].second, 0));
        };
#pragma unroll
        for (int s = 0; s < kAtOnce; ++s) fetch(threadIdx.x + s * kThreads, s);
        if (row >= a.cu_q[a.B]) return;
        const int i = owner_by_wave(a.cu_q, a.B, row), j = row - a.cu_q[i];
        const long long t = (long long)a.ctx[i] + j;
        long long pos = t;
        if (a.positions) pos = a.positions[row];
        if (a.tree) {  // the depth in the tree
            pos = (long long)a.ctx[i] - 1;
            for (int w = 0; w < a.tree_words; ++w) pos += __popcll(a.tree[(size_t)row * a.tree_words + w]);
        }
        pos = pos < 0 ? 0 : pos >= a.T ? a.T - 1 : pos;
        bool stored = t >= 0 && t < (long long)a.max_pages * a.P;  // there is a page for this position
        size_t slot = 0, head_step = 0;
        if (stored) {
            const int pg = (int)(t / a.P), in = (int)(t - (long long)pg * a.P);
            const int page = a.bt[(size_t)i * a.max_pages + pg];
            stored = page >= 0 && page < a.n_pages;  // never write outside the pool
            slot = a.token_major ? ((size_t)page * a.P + in) * a.H_kv : (size_t)page * a.H_kv * a.P + in;
            head_step = a.token_major ? 1 : a.P;
        }
        const float* table = a.cos_sin + (size_t)pos * a.R;
        auto finish = [&](int s) __attribute__((always_inline)) {
            const At p = at[s];
            float u[8], w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                u[k] = PAIRS ? (k < 4 ? x[s].get(2 * k) : y[s].get(2 * k - 8)) : x[s].get(k);
                w[k] = PAIRS ? (k < 4 ? x[s].get(2 * k + 1) : y[s].get(2 * k - 7)) : y[s].get(k);
            }
            if (p.second >= 0) {
                Eight<float> c, n;
                c.load(table + p.turn);
                n.load(table + a.R / 2 + p.turn);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float turned = u[k] * c.get(k) - w[k] * n.get(k);
                    w[k] = w[k] * c.get(k) + u[k] * n.get(k);
                    u[k] = turned;
                }
                if (PAIRS) {
                    float lo[8], hi[8];
#pragma unroll
                    for (int k = 0; k < 4; ++k) { lo[2 * k] = u[k]; lo[2 * k + 1] = w[k]; hi[2 * k] = u[k + 4]; hi[2 * k + 1] = w[k + 4]; }
#pragma unroll
                    for (int k = 0; k < 8; ++k) { u[k] = lo[k]; w[k] = hi[k]; }
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) u[k] = x[s].get(k);
            }
            if (p.part != 0 && !stored) return;
            if (KV8 && p.part != 0) {  // from the fp32 value: one rounding
                const float scale = (p.part == 1 ? a.k_scale : a.v_scale)[p.head];
                uint8_t* to = (uint8_t*)(p.part == 1 ? a.k_cache : a.v_cache) + (slot + p.head * head_step) * a.D;
                auto put = [&](const float* v, int first) {
                    uint32_t o[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        o[k] = pack_e4m3(v[4 * k + 2] / scale, v[4 * k + 3] / scale, pack_e4m3(v[4 * k] / scale, v[4 * k + 1] / scale, 0u, false), true);
                    *reinterpret_cast<u32x2*>(to + first) = u32x2{o[0], o[1]};
                };
                put(u, p.first);
                if (p.second >= 0) put(w, p.second);
                return;
            }
            T* to = p.part == 0 ? (T*)a.q_out + ((size_t)row * a.H_q + p.head) * a.D
                                : (T*)(p.part == 1 ? a.k_cache : a.v_cache) + (slot + p.head * head_step) * a.D;
            if (p.second >= 0) {
                x[s].set(u);
                y[s].set(w);
                y[s].store(to + p.second);
            }
            x[s].store(to + p.first);  // (what is only moved keeps its bits)
        };
        for (int n = threadIdx.x; n < a.pieces;) {
#pragma unroll
            for (int s = 0; s < kAtOnce; ++s)
                if (n + s * kThreads < a.pieces) finish(s);
            n += kAtOnce * kThreads;
            if (n < a.pieces)
#pragma unroll
                for (int s = 0; s < kAtOnce; ++s) fetch(n + s * kThreads, s);
        }
    }
}

template <typename T, bool KV8>
void launch(const RopeArgs& a, bool pairs, void* stream) {
    const dim3 grid((unsigned)std::min(a.N_cap, kMaxRows)), block(kThreads);
    if (pairs) hipLaunchKernelGGL((rope_append_kernel<T, true, KV8>), grid, block, 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL((rope_append_kernel<T, false, KV8>), grid, block, 0, (hipStream_t)stream, a);
}

int append(const char* who, bool kv8, const void* q, const void* k_new, const void* v_new, const float* cos_sin, const int32_t* positions,
           const uint64_t* tree_mask, void* q_out, void* k_cache, void* v_cache, const float* k_scale, const float* v_scale, const int32_t* block_tables,
           const int32_t* ctx_lens, const int32_t* cu_q, const fsr_rope_params* p, void* stream) {
    if (!p) return fail(FSR_EINVAL, "%s: params is null", who);
    if (p->B < 0 || p->N_cap < 0 || p->H_q <= 0 || p->H_kv <= 0 || p->D <= 0 || p->P <= 0 || p->max_pages <= 0 || p->n_pages <= 0 || p->T <= 0)
        return fail(FSR_EINVAL, "%s: B=%d N_cap=%d H_q=%d H_kv=%d D=%d P=%d max_pages=%d n_pages=%d T=%d", who, p->B, p->N_cap, p->H_q, p->H_kv, p->D, p->P,
                    p->max_pages, p->n_pages, p->T);
    if (p->dtype != FSR_BF16 && (kv8 || p->dtype != FSR_F32)) return fail(FSR_EUNSUP, "%s: dtype=%d", who, p->dtype);
    if (p->kv_layout != FSR_KV_HEAD_MAJOR && p->kv_layout != FSR_KV_TOKEN_MAJOR) return fail(FSR_EINVAL, "%s: kv_layout=%d", who, p->kv_layout);
    if ((p->pairs != 0 && p->pairs != 1) || p->reserved != 0) return fail(FSR_EINVAL, "%s: pairs=%d (0 or 1) reserved=%d (0)", who, p->pairs, p->reserved);
    if (p->R <= 0 || p->R > p->D) return fail(FSR_ESHAPE, "%s: R=%d must be 1 .. D=%d", who, p->R, p->D);
    if (p->R % 16 != 0 || p->D % (kv8 ? 16 : 8) != 0 || p->D > 8192)
        return fail(FSR_EUNSUP, "%s: R=%d D=%d (R a multiple of 16, D of %d up to 8192)", who, p->R, p->D, kv8 ? 16 : 8);
    if (p->H_q > 65535 || p->H_kv > 65535 || (long long)(p->H_q + 2LL * p->H_kv) * (p->D / 8) > (1 << 28)) return fail(FSR_EUNSUP, "%s: H_q=%d H_kv=%d D=%d are too large", who, p->H_q, p->H_kv, p->D);
    const int elem = p->dtype == FSR_F32 ? 4 : 2;
    const long long q_row = (long long)p->H_q * p->D, kv_row = (long long)p->H_kv * p->D;
    if (p->q_stride < q_row || p->k_stride < kv_row || p->v_stride < kv_row)
        return fail(FSR_ESHAPE, "%s: rows overlap (q_stride=%lld k_stride=%lld v_stride=%lld elements)", who, (long long)p->q_stride, (long long)p->k_stride, (long long)p->v_stride);
    if ((p->q_stride * elem | p->k_stride * elem | p->v_stride * elem) & 15)
        return fail(FSR_EINVAL, "%s: rows must be a multiple of 16 bytes apart", who);
    if (positions && tree_mask) return fail(FSR_EINVAL, "%s: positions and tree_mask exclude each other", who);
    if (tree_mask && (p->tree_words <= 0 || p->tree_words > FSR_TREE_WORDS_MAX)) return fail(FSR_EINVAL, "%s: tree_words=%d must be 1 .. %d", who, p->tree_words, FSR_TREE_WORDS_MAX);
    if (p->B == 0 || p->N_cap == 0) return FSR_OK;
    if (!q || !k_new || !v_new || !cos_sin || !q_out || !k_cache || !v_cache || !block_tables || !ctx_lens || !cu_q || (kv8 && (!k_scale || !v_scale)))
        return fail(FSR_EINVAL, "%s: null pointer among q/k_new/v_new/cos_sin/q_out/k_cache/v_cache/%sblock_tables/ctx_lens/cu_q", who, kv8 ? "k_scale/v_scale/" : "");
    if (((uintptr_t)q | (uintptr_t)k_new | (uintptr_t)v_new | (uintptr_t)cos_sin | (uintptr_t)q_out | (uintptr_t)k_cache | (uintptr_t)v_cache) & 15)
        return fail(FSR_EINVAL, "%s: q/k_new/v_new/cos_sin/q_out/k_cache/v_cache must be 16-byte aligned", who);
    if (q_out == q && p->q_stride != q_row) return fail(FSR_EINVAL, "%s: q_out is dense, q is not: they cannot be the same", who);
    RopeArgs a{};
    a.q = q; a.k_new = k_new; a.v_new = v_new; a.cos_sin = cos_sin; a.positions = positions; a.tree = tree_mask;
    a.q_out = q_out; a.k_cache = k_cache; a.v_cache = v_cache; a.k_scale = k_scale; a.v_scale = v_scale;
    a.bt = block_tables; a.ctx = ctx_lens; a.cu_q = cu_q;
    a.q_stride = p->q_stride; a.k_stride = p->k_stride; a.v_stride = p->v_stride;
    a.B = p->B; a.N_cap = p->N_cap; a.H_q = p->H_q; a.H_kv = p->H_kv; a.D = p->D; a.R = p->R; a.P = p->P;
    a.max_pages = p->max_pages; a.n_pages = p->n_pages; a.T = p->T; a.tree_words = p->tree_words;
    a.token_major = p->kv_layout == FSR_KV_TOKEN_MAJOR;
    a.turned = p->R / 16;
    a.per_head = a.turned + (p->D - p->R) / 8;
    a.q_pieces = p->H_q * a.per_head;
    a.pieces = a.q_pieces + p->H_kv * (a.per_head + p->D / 8);
    if (kv8) launch<uint16_t, true>(a, p->pairs, stream);
    else if (p->dtype == FSR_BF16) launch<uint16_t, false>(a, p->pairs, stream);
    else launch<float, false>(a, p->pairs, stream);
    return check_launch(who);
}

}  // namespace
}  // namespace fsr

using namespace fsr;

extern "C" int fsr_kv_append_rope(const void* q, const void* k_new, const void* v_new, const float* cos_sin, const int32_t* positions, const uint64_t* tree_mask,
                                  void* q_out, void* k_cache, void* v_cache, const int32_t* block_tables, const int32_t* ctx_lens, const int32_t* cu_q,
                                  const fsr_rope_params* p, void* stream) {
    return append("fsr_kv_append_rope", false, q, k_new, v_new, cos_sin, positions, tree_mask, q_out, k_cache, v_cache, nullptr, nullptr, block_tables, ctx_lens,
                  cu_q, p, stream);
}

extern "C" int fsr_kv_append_rope_kv8(const void* q, const void* k_new, const void* v_new, const float* cos_sin, const int32_t* positions, const uint64_t* tree_mask,
                                      void* q_out, void* k_cache, void* v_cache, const float* k_scale, const float* v_scale, const int32_t* block_tables,
                                      const int32_t* ctx_lens, const int32_t* cu_q, const fsr_rope_params* p, void* stream) {
    return append("fsr_kv_append_rope_kv8", true, q, k_new, v_new, cos_sin, positions, tree_mask, q_out, k_cache, v_cache, k_scale, v_scale, block_tables, ctx_lens,
                  cu_q, p, stream);
}
