// Acceptance of trees of drafted tokens: the path on which the target agrees with the drafts, and the move of its keys and values to
// the positions that follow the context.
//
// A tree is given by its rows' bits: a row's parent is the highest of its bits below itself.  fsr_tree_accept looks at all rows at
// once for a child that carries the token which the target chose at its parent (the first one, by an atomic minimum: the result does
// not depend on the order), then walks down from the first row.  One wave a request; bound by a few round trips to memory, then by
// one LDS read per accepted token: 12 rows 2 us, 256 requests of 8-160 rows 4 us.
//
// fsr_kv_commit: path[k] >= k, so that a row moves to the front or stays.  A thread owns 16 bytes of one head for all rows of a
// request: it reads kBatch rows of the path, then writes them, in ascending order.  A write at place k meets no later read: those are
// at places >= k' > k.  Bound by the round trips length -> path -> pages -> rows: 8 heads of 128, up to 8 tokens, 4 requests 5 us,
// 256 (8-bit, 4 MB) 6 us.
#include <algorithm>
#include <cstdint>

#include "common.hpp"
#include "device_utils.hpp"

namespace fsr {
namespace {

constexpr int kRowsMax = 64 * FSR_TREE_WORDS_MAX;

struct AcceptArgs {
    const int32_t* target;
    const int32_t* draft;
    const uint64_t* tree;
    const int32_t* cu_q;
    int32_t* accepted_len;
    int32_t* n_emitted;
    int32_t* emitted;
    int32_t* path;
    uint8_t* keep;
    int B, N_cap, words, S_max;
};

__global__ __launch_bounds__(kWave) void tree_accept_kernel(AcceptArgs a) {
    __shared__ int32_t target[kRowsMax];
    __shared__ int32_t next[kRowsMax];  // first child of a row that carries the target's token; kRowsMax: none
    const int lane = threadIdx.x, i = blockIdx.x;
    const int row0 = min(max(a.cu_q[i], 0), a.N_cap), rows = min(max(a.cu_q[i + 1], row0), a.N_cap) - row0;
    const int n = min(rows, 64 * a.words);  // rows that have a bit
    for (int j = lane; j < n; j += kWave) {
        target[j] = a.target[row0 + j];
        next[j] = kRowsMax;
    }
    __syncthreads();
    for (int j = lane; j < n; j += kWave) {
        int parent = -1;
        for (int w = j >> 6; w >= 0 && parent < 0; --w) {
            uint64_t bits = a.tree[(size_t)(row0 + j) * a.words + w];
            if (w == j >> 6) bits &= (1ull << (j & 63)) - 1;
            if (bits) parent = 64 * w + 63 - __clzll((long long)bits);
        }
        if (parent >= 0 && a.draft[row0 + j] == target[parent]) atomicMin(&next[parent], j);
    }
    __syncthreads();
    int at = 0, count = 0;  // tokens emitted
    const size_t out = (size_t)i * (a.S_max + 1);
    while (n > 0) {  // (a child lies behind its parent: the walk ends)
        if (lane == 0) {
            a.path[out + count] = at;
            a.emitted[out + count] = target[at];
        }
        ++count;
        const int child = __builtin_amdgcn_readfirstlane(next[at]);  // (read by the wave as one: the first lane writes there next)
        if (lane == 0) next[at] = -1;  // (on the path)
        if (child >= n || count > a.S_max) break;
        at = child;
    }
    __syncthreads();
    if (a.keep)
        for (int j = lane; j < rows; j += kWave) a.keep[row0 + j] = j < n && next[j] < 0;
    for (int k = count + lane; k <= a.S_max; k += kWave) a.path[out + k] = a.emitted[out + k] = -1;
    if (lane == 0) {
        a.accepted_len[i] = count - 1;
        a.n_emitted[i] = count;
    }
}

constexpr int kThreads = 256, kBatch = 8;
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;

struct CommitArgs {
    char* k_cache;
    char* v_cache;
    const int32_t* bt;
    const int32_t* ctx;
    const int32_t* accepted_len;
    const int32_t* path;
    int B, H_kv, P, p_shift, max_pages, n_pages, token_major, row_bytes, S_max;  // p_shift: log2(P), or -1
    int per, pieces;  // threads of a request, of a head
};

__global__ __launch_bounds__(kThreads) void kv_commit_kernel(CommitArgs a) {
    const uint32_t id = blockIdx.x * (uint32_t)kThreads + threadIdx.x, request = id / (uint32_t)a.per;
    if (request >= (uint32_t)a.B) return;
    const int i = (int)request;
    const uint32_t rest = id - request * (uint32_t)a.per, head = rest / (uint32_t)a.pieces;
    const uint32_t in_row = (rest - head * (uint32_t)a.pieces) * 16;
    const int n = min(a.accepted_len[i], a.S_max);
    const long long ctx = a.ctx[i], end = min((long long)a.max_pages * a.P, 1LL << 31);
    const int32_t* path = a.path + (size_t)i * (a.S_max + 1);
    auto place = [&](long long t, bool& there) {  // byte offset of this thread's piece at position t
        there = there && t >= 0 && t < end;
        const uint32_t at = there ? (uint32_t)t : 0u, pg = a.p_shift >= 0 ? at >> a.p_shift : at / (uint32_t)a.P;  // (in 64 bits sixteen of these took 4 us)
        const int page = a.bt[(size_t)i * a.max_pages + pg];
        there = there && page >= 0 && page < a.n_pages;
        if (!there) return (size_t)0;
        const size_t in = at - pg * (uint32_t)a.P;
        const size_t slot = a.token_major ? ((size_t)page * a.P + in) * a.H_kv + head : ((size_t)page * a.H_kv + head) * a.P + in;
        return slot * a.row_bytes + in_row;
    };
    for (int k0 = 1; k0 <= n; k0 += kBatch) {
        u32x4 k[kBatch], v[kBatch];
        size_t to[kBatch];
        bool moves[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int step = k0 + b, source = path[min(step, a.S_max)];
            moves[b] = step <= n && source > step;
            to[b] = place(ctx + step, moves[b]);
            const size_t from = place(ctx + source, moves[b]);
            if (moves[b]) {
                k[b] = *reinterpret_cast<const u32x4*>(a.k_cache + from);
                v[b] = *reinterpret_cast<const u32x4*>(a.v_cache + from);
            }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b)
            if (moves[b]) {
                *reinterpret_cast<u32x4*>(a.k_cache + to[b]) = k[b];
                *reinterpret_cast<u32x4*>(a.v_cache + to[b]) = v[b];
            }
    }
}

}  // namespace
}  // namespace fsr

using namespace fsr;

extern "C" int fsr_tree_accept(const int32_t* target_tokens, const int32_t* draft_tokens, const uint64_t* tree_mask, const int32_t* cu_q, int32_t* accepted_len,
                               int32_t* n_emitted, int32_t* emitted, int32_t* path, uint8_t* keep_mask, const fsr_tree_params* p, void* stream) {
    const char* who = "fsr_tree_accept";
    if (!p) return fail(FSR_EINVAL, "%s: params is null", who);
    if (p->B < 0 || p->N_cap < 0 || p->S_max < 0 || p->reserved != 0) return fail(FSR_EINVAL, "%s: B=%d N_cap=%d S_max=%d reserved=%d", who, p->B, p->N_cap, p->S_max, p->reserved);
    if (p->tree_words <= 0 || p->tree_words > FSR_TREE_WORDS_MAX) return fail(FSR_EINVAL, "%s: tree_words=%d must be 1 .. %d", who, p->tree_words, FSR_TREE_WORDS_MAX);
    if (p->B == 0) return FSR_OK;
    if (!cu_q || !accepted_len || !n_emitted || !emitted || !path || (p->N_cap > 0 && (!target_tokens || !draft_tokens || !tree_mask)))
        return fail(FSR_EINVAL, "%s: null pointer among target_tokens/draft_tokens/tree_mask/cu_q/accepted_len/n_emitted/emitted/path", who);
    AcceptArgs a{};
    a.target = target_tokens; a.draft = draft_tokens; a.tree = tree_mask; a.cu_q = cu_q;
    a.accepted_len = accepted_len; a.n_emitted = n_emitted; a.emitted = emitted; a.path = path; a.keep = keep_mask;
    a.B = p->B; a.N_cap = p->N_cap; a.words = p->tree_words; a.S_max = p->S_max;
    if (p->B > (1 << 25)) return fail(FSR_EUNSUP, "%s: B=%d exceeds 2^25", who, p->B);
    hipLaunchKernelGGL(tree_accept_kernel, dim3((unsigned)p->B), dim3(kWave), 0, (hipStream_t)stream, a);
    return check_launch(who);
}

extern "C" int fsr_kv_commit(void* k_cache, void* v_cache, const int32_t* block_tables, const int32_t* ctx_lens, const int32_t* accepted_len, const int32_t* path,
                             const fsr_commit_params* p, void* stream) {
    const char* who = "fsr_kv_commit";
    if (!p) return fail(FSR_EINVAL, "%s: params is null", who);
    if (p->B < 0 || p->H_kv <= 0 || p->row_bytes <= 0 || p->P <= 0 || p->max_pages <= 0 || p->n_pages <= 0 || p->S_max < 0)
        return fail(FSR_EINVAL, "%s: B=%d H_kv=%d row_bytes=%d P=%d max_pages=%d n_pages=%d S_max=%d", who, p->B, p->H_kv, p->row_bytes, p->P, p->max_pages, p->n_pages, p->S_max);
    if (p->kv_layout != FSR_KV_HEAD_MAJOR && p->kv_layout != FSR_KV_TOKEN_MAJOR) return fail(FSR_EINVAL, "%s: kv_layout=%d", who, p->kv_layout);
    if (p->row_bytes % 16 != 0) return fail(FSR_EUNSUP, "%s: row_bytes=%d, need a multiple of 16", who, p->row_bytes);
    if (p->B == 0 || p->S_max == 0) return FSR_OK;
    if (!k_cache || !v_cache || !block_tables || !ctx_lens || !accepted_len || !path)
        return fail(FSR_EINVAL, "%s: null pointer among k_cache/v_cache/block_tables/ctx_lens/accepted_len/path", who);
    if (((uintptr_t)k_cache | (uintptr_t)v_cache) & 15) return fail(FSR_EINVAL, "%s: k_cache/v_cache must be 16-byte aligned", who);
    CommitArgs a{};
    a.k_cache = (char*)k_cache; a.v_cache = (char*)v_cache;
    a.bt = block_tables; a.ctx = ctx_lens; a.accepted_len = accepted_len; a.path = path;
    a.B = p->B; a.H_kv = p->H_kv; a.P = p->P; a.max_pages = p->max_pages; a.n_pages = p->n_pages;
    a.token_major = p->kv_layout == FSR_KV_TOKEN_MAJOR;
    a.row_bytes = p->row_bytes; a.S_max = p->S_max;
    a.p_shift = (p->P & (p->P - 1)) == 0 ? __builtin_ctz((unsigned)p->P) : -1;
    const long long per = (long long)p->H_kv * (p->row_bytes / 16), blocks = (p->B * per + kThreads - 1) / kThreads;
    if (per > 0x7fffffffLL || blocks > (1 << 23)) return fail(FSR_EUNSUP, "%s: B * H_kv * row_bytes is too large for one launch", who);
    a.per = (int)per;
    a.pieces = p->row_bytes / 16;
    hipLaunchKernelGGL(kv_commit_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a);
    return check_launch(who);
}
