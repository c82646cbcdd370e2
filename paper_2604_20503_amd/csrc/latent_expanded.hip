// Latent attention in its expanded form: keys and values of every head have been computed from the latents (by the caller's
// up-projection), the position part of a key is one row that all heads share:
//     z[j, t] = scale * (q_nope[j] . k_nope[t, h] + q_rope[j] . k_rope[t]).
// Per row and key it costs D_nope + D_rope + D_v multiply-adds a head where the form in the latent's space costs
// 2 D_latent + D_rope, which is worth the up-projection once a request has many rows (a chunk of a prompt).
// Measured: 2048 rows behind 6000 tokens, 32 heads: 314-341 us by card, 938-864 TFLOP/s; 4 prompts of 200-700 rows, 16 heads: 67-69 us, 381-372
// TFLOP/s.  fp32: 2 prompts of 200-700 rows behind up to 1000 keys, 16 heads: 156 us, 47 TFLOP/s of 150.
#include "row_tiles.hpp"

namespace fsr {
namespace {

using namespace row_tiles;

int check(const fsr_expanded_params* p, const char* who) {
    if (!p) return fail(FSR_EINVAL, "%s: params is null", who);
    if (p->B < 0 || p->N_cap < 0 || p->T_cap < 0 || p->H <= 0 || p->max_q_len < 0 || p->max_workgroups < 0)
        return fail(FSR_EINVAL, "%s: B=%d N_cap=%d T_cap=%d H=%d max_q_len=%d max_workgroups=%d", who, p->B, p->N_cap, p->T_cap, p->H, p->max_q_len,
                    p->max_workgroups);
    if (!((p->D_nope == 128 && p->D_rope == 64 && p->D_v == 128) || (p->D_nope == 64 && p->D_rope == 32 && p->D_v == 64)))
        return fail(FSR_EUNSUP, "%s: D_nope=%d D_rope=%d D_v=%d (128/64/128 and 64/32/64 are built)", who, p->D_nope, p->D_rope, p->D_v);
    if (p->dtype != FSR_F32 && p->dtype != FSR_BF16) return fail(FSR_EUNSUP, "%s: dtype=%d", who, p->dtype);
    if (p->out_dtype != FSR_F32 && !(p->out_dtype == FSR_BF16 && p->dtype == FSR_BF16))
        return fail(FSR_EUNSUP, "%s: out_dtype=%d with dtype=%d", who, p->out_dtype, p->dtype);
    if (!(p->scale > 0.0f) || p->scale > 2.0e38f) return fail(FSR_EINVAL, "%s: scale=%g must be > 0 and finite", who, (double)p->scale);
    if (p->B > 65535 || p->H > 65535) return fail(FSR_EUNSUP, "%s: B and H are limited to 65535", who);
    if (p->N_cap > (1 << 30) || p->T_cap > (1 << 30)) return fail(FSR_EUNSUP, "%s: N_cap and T_cap are limited to 2^30 rows", who);
    if (p->reserved != 0) return fail(FSR_EINVAL, "%s: reserved=%d must be 0", who, p->reserved);
    return FSR_OK;
}

int rows_cap(const fsr_expanded_params* p) { return std::max(1, std::min(p->N_cap, kTileRows)); }

template <int DN, int DR, int DV>
int run(const Args& a, const fsr_expanded_params* p, void* stream, const char* who) {
    if (p->dtype == FSR_F32) return launch<Simple<kExpanded, DN, DR, DV>>(a, p->max_workgroups, stream, who);
    if (p->out_dtype == FSR_F32) return launch<Tiled<kExpanded, DN, DR, DV, float, true>>(a, p->max_workgroups, stream, who);
    return launch<Tiled<kExpanded, DN, DR, DV, uint16_t, true>>(a, p->max_workgroups, stream, who);
}

}  // namespace
}  // namespace fsr

using namespace fsr;

extern "C" int fsr_expanded_workspace_bytes(const fsr_expanded_params* p, size_t* out_bytes) {
    int rc = check(p, "fsr_expanded_workspace_bytes");
    if (rc != FSR_OK) return rc;
    if (!out_bytes) return fail(FSR_EINVAL, "fsr_expanded_workspace_bytes: out_bytes is null");
    *out_bytes = layout_of(rows_cap(p), p->D_v, 0, false).total;
    return FSR_OK;
}

extern "C" int fsr_latent_attention_expanded(const void* q, const void* kv, const void* k_rope, const int32_t* cu_q, const int32_t* cu_k, void* out,
                                             float* lse, const fsr_expanded_params* p, void* workspace, size_t ws_bytes, void* stream) {
    const char* who = "fsr_latent_attention_expanded";
    int rc = check(p, who);
    if (rc != FSR_OK) return rc;
    if (p->B == 0 || p->N_cap == 0) return FSR_OK;
    if (!q || !cu_q || !cu_k || !out || (p->T_cap > 0 && (!kv || !k_rope))) return fail(FSR_EINVAL, "%s: null pointer among q/kv/k_rope/cu_q/cu_k/out", who);
    if (((uintptr_t)q | (uintptr_t)kv | (uintptr_t)k_rope | (uintptr_t)out) & 15) return fail(FSR_EINVAL, "%s: q/kv/k_rope/out must be 16-byte aligned", who);
    const Layout l = layout_of(rows_cap(p), p->D_v, 0, false);
    if (!workspace || ws_bytes < l.total) return fail(FSR_EWS, "%s: workspace %zu bytes, need %zu", who, ws_bytes, l.total);
    if ((uintptr_t)workspace & 255) return fail(FSR_EWS, "%s: workspace must be 256-byte aligned", who);
    Args a{};
    const long long elem = p->dtype == FSR_F32 ? 4 : 2, row = (p->D_nope + p->D_v) * elem;
    a.q = q;
    a.k_head = (const char*)kv;
    a.k_tail = (const char*)k_rope;
    a.v = (const char*)kv + p->D_nope * elem;
    a.cu_q = cu_q; a.cu_k = cu_k;
    a.out = out; a.lse = lse;
    a.B = p->B; a.N_cap = p->N_cap; a.T_cap = p->T_cap; a.H = p->H; a.H_stream = p->H; a.G = 1;
    a.P = 1; a.max_pages = 1; a.n_pages = 1;
    a.head_stride = a.v_stride = (uint32_t)(p->H * row);
    a.tail_stride = (uint32_t)(p->D_rope * elem);
    a.head_hk = a.v_hk = row;
    a.scale = p->scale;
    a.scale_log2 = p->scale * kLog2e;
    a.m_cap = rows_cap(p);
    place(a, l, workspace);
    return p->D_nope == 128 ? run<128, 64, 128>(a, p, stream, who) : run<64, 32, 64>(a, p, stream, who);
}
