// Latent caches: every token of a request stores one row that all query heads share, the latent vector (from which keys and
// values of all heads are linear images) followed by the key part that carries the position.  The rows of a call enter the
// paged cache before its attention (fsr_latent_append), come back as contiguous rows for the expanded form
// (fsr_latent_gather), and are attended over directly by queries that have been taken into the latent's space
// (fsr_latent_attention).
#include "latent_tiles.hpp"

namespace fsr {
namespace {

using namespace row_tiles;

// ---------------------------------------------------------------------------------------------------------------
// append and gather: 16 bytes per thread and step.  A workgroup takes kMoveRows consecutive rows: their owners and slots are
// looked up once, by a lane each, and not by every thread that moves a piece of a row.
// Bound by memory: 96 contexts of 512-8192 rows of 576 bytes come back at 4.6 TB/s where a copy reaches 5.1; 4 rows take a launch, 3 us.
// ---------------------------------------------------------------------------------------------------------------
constexpr int kMoveRows = 32;

struct MoveArgs {
    char* cache;
    char* latent;
    char* rope;
    const int32_t* bt;
    const int32_t* ctx;  // append: position of a request's first row; gather: null, position 0
    const int32_t* cu;
    int B, rows_cap, P, max_pages, n_pages;
    int row0;            // first row of the launch
    int head16, tail16;  // 16-byte pieces of a latent and of a rope part
};

template <bool APPEND>
__global__ __launch_bounds__(kThreads) void move_rows_kernel(MoveArgs a) {
    __shared__ long long slots[kMoveRows];  // -1: no such row, or nowhere to put it
    const int row0 = a.row0 + blockIdx.x * kMoveRows;
    if (threadIdx.x < kMoveRows) {
        const int row = row0 + threadIdx.x;
        long long slot = -1;
        if (row < a.rows_cap && row >= a.cu[0] && row < a.cu[a.B]) {
            int lo = 0, hi = a.B;  // largest i with cu[i] <= row
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (a.cu[mid] <= row) lo = mid; else hi = mid;
            }
            const long long t = (long long)(APPEND ? a.ctx[lo] : 0) + (row - a.cu[lo]);
            if (t >= 0 && t < (long long)a.max_pages * a.P) {
                const int pg = (int)(t / a.P);
                int page = a.bt[(size_t)lo * a.max_pages + pg];
                // what is read comes from some page of the pool, nothing is written outside of it
                if (!APPEND) page = min(max(page, 0), a.n_pages - 1);
                if (page >= 0 && page < a.n_pages) slot = (long long)page * a.P + (t - (long long)pg * a.P);
            } else if (!APPEND) {
                slot = -2;  // no page: zeros
            }
        }
        slots[threadIdx.x] = slot;
    }
    __syncthreads();
    const int each = a.head16 + a.tail16;
    for (int x = threadIdx.x; x < kMoveRows * each; x += kThreads) {
        const int r = x / each, part = x - r * each;
        const long long slot = slots[r];
        if (slot == -1) continue;
        const size_t row = (size_t)(row0 + r);
        u32x4* out_of_cache = reinterpret_cast<u32x4*>(part < a.head16 ? a.latent + (row * a.head16 + part) * 16 : a.rope + (row * a.tail16 + (part - a.head16)) * 16);
        u32x4* in_cache = reinterpret_cast<u32x4*>(a.cache + ((size_t)slot * each + part) * 16);
        if (APPEND) *in_cache = *out_of_cache;
        else *out_of_cache = slot == -2 ? u32x4{0, 0, 0, 0} : *in_cache;
    }
}

int check_cache(const fsr_latent_params* p, const char* who) {
    if (!p) return fail(FSR_EINVAL, "%s: params is null", who);
    if (p->B < 0 || p->N_cap < 0 || p->D_latent <= 0 || p->D_rope <= 0 || p->P <= 0 || p->max_pages <= 0 || p->n_pages <= 0)
        return fail(FSR_EINVAL, "%s: B=%d N_cap=%d D_latent=%d D_rope=%d P=%d max_pages=%d n_pages=%d", who, p->B, p->N_cap, p->D_latent, p->D_rope, p->P,
                    p->max_pages, p->n_pages);
    if (p->dtype != FSR_F32 && p->dtype != FSR_BF16) return fail(FSR_EUNSUP, "%s: dtype=%d", who, p->dtype);
    const int elem = p->dtype == FSR_F32 ? 4 : 2;
    if ((long long)p->D_latent * elem % 16 != 0 || (long long)p->D_rope * elem % 16 != 0)
        return fail(FSR_EUNSUP, "%s: D_latent=%d and D_rope=%d must each fill whole pieces of 16 bytes", who, p->D_latent, p->D_rope);
    if (p->D_latent > 8192 || p->D_rope > 8192) return fail(FSR_EUNSUP, "%s: D_latent=%d D_rope=%d exceed 8192", who, p->D_latent, p->D_rope);
    if (p->reserved != 0) return fail(FSR_EINVAL, "%s: reserved=%d must be 0", who, p->reserved);
    return FSR_OK;
}

int move_rows(bool append, void* cache, void* latent, void* rope, const int32_t* bt, const int32_t* ctx, const int32_t* cu, const fsr_latent_params* p,
              int rows_cap, void* stream, const char* who) {
    if (((uintptr_t)cache | (uintptr_t)latent | (uintptr_t)rope) & 15) return fail(FSR_EINVAL, "%s: cache, latent and rope rows must be 16-byte aligned", who);
    MoveArgs a;
    const int elem = p->dtype == FSR_F32 ? 4 : 2;
    a.cache = (char*)cache; a.latent = (char*)latent; a.rope = (char*)rope;
    a.bt = bt; a.ctx = ctx; a.cu = cu;
    a.B = p->B; a.rows_cap = rows_cap; a.P = p->P; a.max_pages = p->max_pages; a.n_pages = p->n_pages;
    a.head16 = p->D_latent * elem / 16; a.tail16 = p->D_rope * elem / 16;
    constexpr long long kMost = (long long)kMaxBlocks * kMoveRows;
    for (long long first = 0; first < rows_cap; first += kMost) {
        a.row0 = (int)first;
        const dim3 grid((unsigned)((std::min(rows_cap - first, kMost) + kMoveRows - 1) / kMoveRows));
        if (append) hipLaunchKernelGGL(move_rows_kernel<true>, grid, dim3(kThreads), 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL(move_rows_kernel<false>, grid, dim3(kThreads), 0, (hipStream_t)stream, a);
    }
    return check_launch(who);
}

// ---------------------------------------------------------------------------------------------------------------
// attention in the latent's space
// ---------------------------------------------------------------------------------------------------------------
int check_attention(const fsr_latent_params* p, const char* who) {
    int rc = check_cache(p, who);
    if (rc != FSR_OK) return rc;
    if (p->H <= 0 || p->max_q_len < 0 || p->max_workgroups < 0)
        return fail(FSR_EINVAL, "%s: H=%d max_q_len=%d max_workgroups=%d", who, p->H, p->max_q_len, p->max_workgroups);
    if ((p->D_latent != 256 && p->D_latent != 512) || (p->D_rope != 32 && p->D_rope != 64))
        return fail(FSR_EUNSUP, "%s: D_latent=%d D_rope=%d (256 or 512, and 32 or 64, are built)", who, p->D_latent, p->D_rope);
    if (p->out_dtype != FSR_F32 && !(p->out_dtype == FSR_BF16 && p->dtype == FSR_BF16))
        return fail(FSR_EUNSUP, "%s: out_dtype=%d with dtype=%d", who, p->out_dtype, p->dtype);
    if (!(p->scale > 0.0f) || p->scale > 2.0e38f) return fail(FSR_EINVAL, "%s: scale=%g must be > 0 and finite", who, (double)p->scale);
    if (p->B > 65535 || p->H > 65535) return fail(FSR_EUNSUP, "%s: B and H are limited to 65535", who);
    if ((long long)p->N_cap * p->H > (1LL << 30)) return fail(FSR_EUNSUP, "%s: N_cap * H exceeds 2^30 rows", who);
    if ((long long)p->max_pages * p->P > (1LL << 30)) return fail(FSR_EUNSUP, "%s: max_pages * P exceeds 2^30 tokens", who);
    if ((long long)p->n_pages * p->P > 0xffffffffLL) return fail(FSR_EUNSUP, "%s: n_pages * P exceeds 2^32 slots", who);
    return FSR_OK;
}

int rows_cap(const fsr_latent_params* p) { return (int)std::max(1LL, std::min((long long)p->N_cap * p->H, 64LL)); }  // (both kernels' tiles)

template <int DL, int DR>
int run(const Args& a, const fsr_latent_params* p, void* stream, const char* who) {
    if (p->dtype == FSR_F32) return launch<Simple<kLatent, DL, DR, DL>>(a, p->max_workgroups, stream, who);
    const bool pages16 = p->P % 16 == 0;
    if (p->out_dtype == FSR_F32)
        return pages16 ? launch<Latent<DL, DR, float, true>>(a, p->max_workgroups, stream, who) : launch<Latent<DL, DR, float, false>>(a, p->max_workgroups, stream, who);
    return pages16 ? launch<Latent<DL, DR, uint16_t, true>>(a, p->max_workgroups, stream, who) : launch<Latent<DL, DR, uint16_t, false>>(a, p->max_workgroups, stream, who);
}

}  // namespace
}  // namespace fsr

using namespace fsr;

extern "C" int fsr_latent_append(const void* latent_new, const void* rope_new, void* cache, const int32_t* block_tables, const int32_t* ctx_lens,
                                 const int32_t* cu_q, const fsr_latent_params* p, void* stream) {
    int rc = check_cache(p, "fsr_latent_append");
    if (rc != FSR_OK) return rc;
    if (p->B == 0 || p->N_cap == 0) return FSR_OK;
    if (!latent_new || !rope_new || !cache || !block_tables || !ctx_lens || !cu_q)
        return fail(FSR_EINVAL, "fsr_latent_append: null pointer among latent_new/rope_new/cache/block_tables/ctx_lens/cu_q");
    return move_rows(true, cache, const_cast<void*>(latent_new), const_cast<void*>(rope_new), block_tables, ctx_lens, cu_q, p, p->N_cap, stream,
                     "fsr_latent_append");
}

extern "C" int fsr_latent_gather(const void* cache, const int32_t* block_tables, const int32_t* cu_k, void* latent_out, void* rope_out,
                                 const fsr_latent_params* p, void* stream) {
    int rc = check_cache(p, "fsr_latent_gather");
    if (rc != FSR_OK) return rc;
    if (p->B == 0 || p->N_cap == 0) return FSR_OK;
    if (!cache || !block_tables || !cu_k || !latent_out || !rope_out)
        return fail(FSR_EINVAL, "fsr_latent_gather: null pointer among cache/block_tables/cu_k/latent_out/rope_out");
    return move_rows(false, const_cast<void*>(cache), latent_out, rope_out, block_tables, nullptr, cu_k, p, p->N_cap, stream, "fsr_latent_gather");
}

extern "C" int fsr_latent_workspace_bytes(const fsr_latent_params* p, size_t* out_bytes) {
    int rc = check_attention(p, "fsr_latent_workspace_bytes");
    if (rc != FSR_OK) return rc;
    if (!out_bytes) return fail(FSR_EINVAL, "fsr_latent_workspace_bytes: out_bytes is null");
    *out_bytes = layout_of(rows_cap(p), p->D_latent, 0, false).total;
    return FSR_OK;
}

extern "C" int fsr_latent_attention(const void* q, const void* cache, const int32_t* block_tables, const int32_t* ctx_lens, const int32_t* cu_q, void* out,
                                    float* lse, const fsr_latent_params* p, void* workspace, size_t ws_bytes, void* stream) {
    const char* who = "fsr_latent_attention";
    int rc = check_attention(p, who);
    if (rc != FSR_OK) return rc;
    if (p->B == 0 || p->N_cap == 0) return FSR_OK;
    if (!q || !cache || !block_tables || !ctx_lens || !cu_q || !out) return fail(FSR_EINVAL, "%s: null pointer among q/cache/block_tables/ctx_lens/cu_q/out", who);
    if (((uintptr_t)q | (uintptr_t)cache | (uintptr_t)out) & 15) return fail(FSR_EINVAL, "%s: q/cache/out must be 16-byte aligned", who);
    const Layout l = layout_of(rows_cap(p), p->D_latent, 0, false);
    if (!workspace || ws_bytes < l.total) return fail(FSR_EWS, "%s: workspace %zu bytes, need %zu", who, ws_bytes, l.total);
    if ((uintptr_t)workspace & 255) return fail(FSR_EWS, "%s: workspace must be 256-byte aligned", who);
    Args a{};
    const long long elem = p->dtype == FSR_F32 ? 4 : 2, row = (p->D_latent + p->D_rope) * elem;
    a.q = q;
    a.k_head = (const char*)cache;
    a.k_tail = (const char*)cache + p->D_latent * elem;
    a.v = (const char*)cache;
    a.bt = block_tables; a.ctx = ctx_lens; a.cu_q = cu_q;
    a.out = out; a.lse = lse;
    a.B = p->B; a.N_cap = p->N_cap; a.H = p->H; a.H_stream = 1; a.G = p->H;
    a.P = p->P; a.max_pages = p->max_pages; a.n_pages = p->n_pages;
    a.p_shift = (p->P & (p->P - 1)) == 0 ? __builtin_ctz((unsigned)p->P) : -1;
    a.page_slots = (uint32_t)p->P;
    a.head_stride = a.tail_stride = a.v_stride = (uint32_t)row;
    a.scale = p->scale;
    a.scale_log2 = p->scale * kLog2e;
    a.m_cap = rows_cap(p);
    place(a, l, workspace);
    if (p->D_latent == 512) return p->D_rope == 64 ? run<512, 64>(a, p, stream, who) : run<512, 32>(a, p, stream, who);
    return p->D_rope == 64 ? run<256, 64>(a, p, stream, who) : run<256, 32>(a, p, stream, who);
}
