// Cache append with the position rotation on the way: a call's query and key rows are turned to their positions, keys and values enter
// the request's pages.
//     first R elements of a head, pairs (a, b) = (x[i], x[i + R/2]) or (x[2i], x[2i + 1]):   a cos - b sin,  b cos + a sin
// Memory-bound: every element is read once and written once.  A workgroup takes a row.  A thread takes the same 16 elements, which are
// rotated with each other, of several heads (or 8 that are only moved), so that its cosines stay in registers and places need no divisions.
// Its first loads go out before the row's request, page and position are known (four round trips to memory one after the other: offsets,
// length and table, cosines).  2891 rows of 64/8 heads of 128 into 8-bit caches (114 MB): 21.7 us, 5.3 TB/s, where a copy of 1 GiB reaches
// 5.1; 8 rows: 4 us, those round trips and a launch.
#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "common.hpp"
#include "device_utils.hpp"

namespace fsr {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxRows = 1 << 22;   // of a launch, a workgroup each

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
    int B, N_cap, H_q, H_kv, D, R, P, p_shift, max_pages, n_pages, T, tree_words, token_major;
    int turned, per_head;  // pieces of a head that are rotated, of a head
    int lanes, step;       // threads of a head, heads at once
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

// x / scale as fp32 rounds it.  The quotient by the rounded inverse is off by a unit at most, and one step of Newton's method, whose
// residual an fma gives exactly, rounds it as the division would (3 instructions, not 10): for scales of ordinary size, but for those whose
// fraction is all ones.
struct Divisor {
    float scale, inverse;
    bool plain;
    __device__ __forceinline__ void set(float s) {
        scale = s;
        inverse = 1.0f / s;
        plain = !(fabsf(s) > 1e-15f && fabsf(s) < 1e30f) || (__builtin_bit_cast(uint32_t, s) & 0x7fffffu) == 0x7fffffu;
    }
    __device__ __forceinline__ float of(float x) const {
        if (plain) return x / scale;
        const float q = x * inverse, better = fmaf(fmaf(-q, scale, x), inverse, q);
        return fabsf(q) < INFINITY && fabsf(x) > 1e-30f ? better : q;  // (the residual of a smaller x is below fp32; its code is 0)
    }
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

template <typename T, bool PAIRS, bool KV8>
__global__ __launch_bounds__(kThreads) void rope_append_kernel(RopeArgs a) {
    const int row = blockIdx.x, heads = a.H_q + 2 * a.H_kv;
    const int lane_head = (int)((uint32_t)threadIdx.x / (uint32_t)a.lanes), lane = threadIdx.x - lane_head * a.lanes;
    const bool idle = lane_head >= a.step;  // (threads that are left over where a head's pieces do not divide their number)
    const T* const from_q = (const T*)a.q + row * a.q_stride;
    const T* const from_k = (const T*)a.k_new + row * a.k_stride;
    const T* const from_v = (const T*)a.v_new + row * a.v_stride;
    int first = 0, second = 0;  // the thread's elements of every head; second < 0: eight that are moved as they are
    auto place_piece = [&](int u) __attribute__((always_inline)) {
        if (u < a.turned) {
            first = PAIRS ? 16 * u : 8 * u;
            second = PAIRS ? 16 * u + 8 : 8 * u + a.R / 2;
        } else {
            first = a.R + 8 * (u - a.turned);
            second = -1;
        }
    };
    Eight<T> x, y;  // of one head: the next one's loads go out when it is stored (with two heads at once 371 MB took 84 us, not 78)
    auto fetch = [&](int h) __attribute__((always_inline)) {
        if (idle || h >= heads) return;
        const T* at = h < a.H_q ? from_q + h * a.D : h < a.H_q + a.H_kv ? from_k + (h - a.H_q) * a.D : from_v + (h - a.H_q - a.H_kv) * a.D;
        x.load(at + first);
        if (second >= 0) y.load(at + second);
    };
    place_piece(lane);
    fetch(lane_head);

    // all of this is the same for the whole workgroup
    if (row < uniform(a.cu_q[0]) || row >= uniform(a.cu_q[a.B])) return;  // (offsets out of a longer list may begin anywhere)
    const int i = uniform(owner_by_wave(a.cu_q, a.B, row)), c = uniform(a.ctx[i]), j = row - uniform(a.cu_q[i]);
    const long long t = (long long)c + j;
    long long pos = t;
    if (a.positions) pos = uniform(a.positions[row]);
    if (a.tree) {  // the depth in the tree
        int bits = 0;
        const uint32_t* words = reinterpret_cast<const uint32_t*>(a.tree + (size_t)row * a.tree_words);
        for (int w = 0; w < 2 * a.tree_words; ++w) bits += __popc((unsigned)uniform((int)words[w]));
        pos = (long long)c + bits - 1;
    }
    const int turn = pos < 0 ? 0 : pos >= a.T ? a.T - 1 : (int)pos;
    bool stored = t >= 0 && t < min((long long)a.max_pages * a.P, 1LL << 31);  // there is a page for this position
    size_t slot = 0, head_step = 0;
    if (stored) {
        const uint32_t pg = a.p_shift >= 0 ? (uint32_t)t >> a.p_shift : (uint32_t)t / (uint32_t)a.P, in = (uint32_t)t - pg * (uint32_t)a.P;
        const int page = uniform(a.bt[(size_t)i * a.max_pages + pg]);
        stored = page >= 0 && page < a.n_pages;  // never write outside the pool
        slot = (a.token_major ? ((size_t)page * a.P + in) * a.H_kv : (size_t)page * a.H_kv * a.P + in) * a.D;
        head_step = (size_t)(a.token_major ? 1 : a.P) * a.D;
    }
    if (idle) return;
    const float* table = a.cos_sin + (size_t)turn * a.R;
    T* const to_q = (T*)a.q_out + (size_t)row * a.H_q * a.D;

    for (int piece = lane; piece < a.per_head; piece += a.lanes) {  // (once, but for heads of more pieces than there are threads)
        Eight<float> cosines, sines;
        if (piece < a.turned) {
            cosines.load(table + 8 * piece);
            sines.load(table + a.R / 2 + 8 * piece);
        }
        if (piece != lane) {
            place_piece(piece);
            fetch(lane_head);
        }
        auto finish = [&](int h) __attribute__((always_inline)) {
            const bool is_q = h < a.H_q, is_k = !is_q && h < a.H_q + a.H_kv;
            const int g = is_q ? h : is_k ? h - a.H_q : h - a.H_q - a.H_kv;
            const bool turns = second >= 0 && (is_q || is_k);
            float u[8], w[8];  // the two of each pair
            if (turns) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float v = PAIRS ? (k < 4 ? x.get(2 * k) : y.get(2 * k - 8)) : x.get(k);
                    const float z = PAIRS ? (k < 4 ? x.get(2 * k + 1) : y.get(2 * k - 7)) : y.get(k);
                    const float turned = v * cosines.get(k) - z * sines.get(k), other = z * cosines.get(k) + v * sines.get(k);
                    if (!PAIRS) {
                        u[k] = turned;
                        w[k] = other;
                    } else if (k < 4) {
                        u[2 * k] = turned;
                        u[2 * k + 1] = other;
                    } else {
                        w[2 * k - 8] = turned;
                        w[2 * k - 7] = other;
                    }
                }
            }
            if (KV8 && !is_q) {  // from the fp32 value: one rounding
                if (!stored) return;
                if (!turns) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        u[k] = x.get(k);
                        w[k] = y.get(k);
                    }
                }
                Divisor scale;
                scale.set((is_k ? a.k_scale : a.v_scale)[g]);
                uint8_t* to = (uint8_t*)(is_k ? a.k_cache : a.v_cache) + slot + g * head_step;
                auto put = [&](const float* v, int at) {
                    uint32_t o[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        o[k] = pack_e4m3(scale.of(v[4 * k + 2]), scale.of(v[4 * k + 3]), pack_e4m3(scale.of(v[4 * k]), scale.of(v[4 * k + 1]), 0u, false), true);
                    *reinterpret_cast<u32x2*>(to + at) = u32x2{o[0], o[1]};
                };
                put(u, first);
                if (second >= 0) put(w, second);
            } else if (is_q || stored) {
                T* to = is_q ? to_q + g * a.D : (T*)(is_k ? a.k_cache : a.v_cache) + slot + g * head_step;
                if (turns) {  // (what is only moved keeps its bits)
                    x.set(u);
                    y.set(w);
                }
                x.store(to + first);
                if (second >= 0) y.store(to + second);
            }
        };
        for (int h = lane_head; h < heads;) {
            finish(h);
            h += a.step;
            fetch(h);
        }
    }
}

template <typename T, bool KV8>
void launch(const RopeArgs& a, bool pairs, void* stream) {
    const dim3 grid((unsigned)a.N_cap), block(kThreads);
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
    if (p->H_q > 65535 || p->H_kv > 65535 || p->N_cap > kMaxRows) return fail(FSR_EUNSUP, "%s: H_q=%d H_kv=%d (up to 65535) N_cap=%d (up to 2^22)", who, p->H_q, p->H_kv, p->N_cap);
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
    a.p_shift = (p->P & (p->P - 1)) == 0 ? __builtin_ctz((unsigned)p->P) : -1;
    a.max_pages = p->max_pages; a.n_pages = p->n_pages; a.T = p->T; a.tree_words = p->tree_words;
    a.token_major = p->kv_layout == FSR_KV_TOKEN_MAJOR;
    a.turned = p->R / 16;
    a.per_head = a.turned + (p->D - p->R) / 8;
    a.lanes = std::min(a.per_head, kThreads);
    a.step = kThreads / a.lanes;
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
