// Verification attention for a batch whose requests share long prefixes (a system prompt, a document asked about many times).
// The rows of all requests of a group attend to the group's prefix in common: its keys and values are read once per KV head
// and 128 packed rows, and their products are matrix-core sized, where request by request every one reads them again.  A
// request's own tokens behind the prefix are a second sequence of the same launch; the two results of a row are joined by
// their softmax statistics.
// Measured: 64 requests of 2-9 rows behind 8192 common tokens and 64-1024 of their own, 32/8 heads of 128: 101-107 us by card; 192 requests in
// 4 groups, 64/8 heads: 490-526 us, 795-741 TFLOP/s.  Own contexts of few rows cost most for what they are: three of four waves only load.
// us beside fsr_verify_attention with a plan, 300 tokens of their own, 32/8 heads, behind 256 / 1024 / 8192 common ones: 8 requests 33 and 19 / 32
// and 23 / 39 and 42; 64 requests 48 and 38 / 57 and 59 / 103 and 324; 64 requests in groups of one 57 and 40 / 96 and 70 / 426 and 366.
#include "row_tiles.hpp"

namespace fsr {
namespace {

using namespace row_tiles;

int check(const fsr_attn_params* p, int n_groups, const char* who) {
    if (!p) return fail(FSR_EINVAL, "%s: params is null", who);
    if (p->B < 0 || p->N_cap < 0 || p->H_q <= 0 || p->H_kv <= 0 || p->max_pages <= 0 || p->n_pages <= 0 || p->P <= 0 || p->max_workgroups < 0 ||
        p->max_q_len < 0 || n_groups < 0 || (p->kv_layout != FSR_KV_HEAD_MAJOR && p->kv_layout != FSR_KV_TOKEN_MAJOR))
        return fail(FSR_EINVAL, "%s: B=%d N_cap=%d H_q=%d H_kv=%d max_pages=%d n_pages=%d P=%d max_workgroups=%d max_q_len=%d n_groups=%d kv_layout=%d", who,
                    p->B, p->N_cap, p->H_q, p->H_kv, p->max_pages, p->n_pages, p->P, p->max_workgroups, p->max_q_len, n_groups, p->kv_layout);
    if (p->H_q % p->H_kv != 0) return fail(FSR_ESHAPE, "%s: H_q=%d is not a multiple of H_kv=%d", who, p->H_q, p->H_kv);
    if (p->D != 64 && p->D != 128) return fail(FSR_EUNSUP, "%s: head dim %d (64 and 128 are built)", who, p->D);
    if (p->dtype != FSR_F32 && p->dtype != FSR_BF16) return fail(FSR_EUNSUP, "%s: dtype=%d", who, p->dtype);
    if (p->out_dtype != FSR_F32 && !(p->out_dtype == FSR_BF16 && p->dtype == FSR_BF16))
        return fail(FSR_EUNSUP, "%s: out_dtype=%d with dtype=%d", who, p->out_dtype, p->dtype);
    if (!(p->scale > 0.0f) || p->scale > 2.0e38f) return fail(FSR_EINVAL, "%s: scale=%g must be > 0 and finite", who, (double)p->scale);
    if (p->B > 65535 || p->H_q > 65535 || n_groups > 65535) return fail(FSR_EUNSUP, "%s: B, H_q and n_groups are limited to 65535", who);
    if ((long long)p->N_cap * p->H_q > (1LL << 30)) return fail(FSR_EUNSUP, "%s: N_cap * H_q exceeds 2^30 rows", who);
    if ((long long)p->max_pages * p->P > (1LL << 30)) return fail(FSR_EUNSUP, "%s: max_pages * P exceeds 2^30 tokens", who);
    if ((long long)p->n_pages * p->P * p->H_kv > 0xffffffffLL) return fail(FSR_EUNSUP, "%s: n_pages * P * H_kv exceeds 2^32 key rows", who);
    return FSR_OK;
}

Layout layout(const fsr_attn_params* p, int& m_cap) {
    m_cap = (int)std::max(1LL, std::min((long long)p->N_cap * (p->H_q / p->H_kv), (long long)kTileRows));
    return layout_of(m_cap, p->D, (long long)p->N_cap * p->H_q, true);
}

template <int D>
int run(const Args& a, const fsr_attn_params* p, void* stream, const char* who) {
    if (p->dtype == FSR_F32) return launch<Simple<kShared, D, 0, D>>(a, p->max_workgroups, stream, who);
    const bool pages16 = p->P % 16 == 0;
    if (p->out_dtype == FSR_F32)
        return pages16 ? launch<Tiled<kShared, D, 0, D, float, true>>(a, p->max_workgroups, stream, who) : launch<Tiled<kShared, D, 0, D, float, false>>(a, p->max_workgroups, stream, who);
    return pages16 ? launch<Tiled<kShared, D, 0, D, uint16_t, true>>(a, p->max_workgroups, stream, who) : launch<Tiled<kShared, D, 0, D, uint16_t, false>>(a, p->max_workgroups, stream, who);
}

}  // namespace
}  // namespace fsr

using namespace fsr;

extern "C" int fsr_shared_workspace_bytes(const fsr_attn_params* p, size_t* out_bytes) {
    int rc = check(p, 0, "fsr_shared_workspace_bytes");
    if (rc != FSR_OK) return rc;
    if (!out_bytes) return fail(FSR_EINVAL, "fsr_shared_workspace_bytes: out_bytes is null");
    int m_cap;
    *out_bytes = layout(p, m_cap).total;
    return FSR_OK;
}

extern "C" int fsr_verify_attention_shared(const void* q, const void* k_cache, const void* v_cache, const int32_t* block_tables, const int32_t* ctx_lens,
                                           const int32_t* cu_q, const int32_t* cu_groups, const int32_t* prefix_lens, int32_t n_groups, void* out,
                                           float* lse, const fsr_attn_params* p, void* workspace, size_t ws_bytes, void* stream) {
    const char* who = "fsr_verify_attention_shared";
    int rc = check(p, n_groups, who);
    if (rc != FSR_OK) return rc;
    if (p->B == 0 || p->N_cap == 0 || n_groups == 0) return FSR_OK;
    if (!q || !k_cache || !v_cache || !block_tables || !ctx_lens || !cu_q || !cu_groups || !prefix_lens || !out)
        return fail(FSR_EINVAL, "%s: null pointer among q/k_cache/v_cache/block_tables/ctx_lens/cu_q/cu_groups/prefix_lens/out", who);
    if (((uintptr_t)q | (uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)out) & 15)
        return fail(FSR_EINVAL, "%s: q/k_cache/v_cache/out must be 16-byte aligned", who);
    Args a{};
    const Layout l = layout(p, a.m_cap);
    if (!workspace || ws_bytes < l.total) return fail(FSR_EWS, "%s: workspace %zu bytes, need %zu", who, ws_bytes, l.total);
    if ((uintptr_t)workspace & 255) return fail(FSR_EWS, "%s: workspace must be 256-byte aligned", who);
    const long long elem = p->dtype == FSR_F32 ? 4 : 2, row = p->D * elem;
    const bool token_major = p->kv_layout == FSR_KV_TOKEN_MAJOR;
    a.q = q;
    a.k_head = (const char*)k_cache;
    a.v = (const char*)v_cache;
    a.bt = block_tables; a.ctx = ctx_lens; a.cu_q = cu_q; a.cu_groups = cu_groups; a.prefix = prefix_lens;
    a.out = out; a.lse = lse;
    a.B = p->B; a.N_cap = p->N_cap; a.H = p->H_q; a.H_stream = p->H_kv; a.G = p->H_q / p->H_kv; a.n_groups = n_groups;
    a.P = p->P; a.max_pages = p->max_pages; a.n_pages = p->n_pages;
    a.p_shift = (p->P & (p->P - 1)) == 0 ? __builtin_ctz((unsigned)p->P) : -1;
    a.page_slots = (uint32_t)(token_major ? p->P : p->P * p->H_kv);
    a.head_stride = a.v_stride = (uint32_t)(token_major ? p->H_kv * row : row);
    a.head_hk = a.v_hk = token_major ? row : p->P * row;
    a.scale = p->scale;
    a.scale_log2 = p->scale * kLog2e;
    place(a, l, workspace);
    return p->D == 128 ? run<128>(a, p, stream, who) : run<64>(a, p, stream, who);
}
