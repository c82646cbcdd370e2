// Log probabilities of given tokens, the entropy and the largest alternatives of rows of logits.
//     x_v = (z_v - m) / T with m the row's largest logit,  S = sum_v exp x_v
//     log p_v = x_v - log S,   H = log S - sum_v exp(x_v) x_v / S
// Differences are taken before they are scaled, so that logits of any size keep their digits; H is a sum of terms of one sign.
#include <algorithm>
#include <cstdint>

#include "common.hpp"
#include "device_utils.hpp"

namespace fsr {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453094;

struct LogprobArgs {
    const void* logits;
    const int32_t* n_rows;
    const int32_t* tokens;
    float* logprobs;
    float* entropy;
    int32_t* top_ids;
    float* top_logprobs;
    long long stride;
    int N_cap, V, M, K;
    float scale;   // log2(e) / T
    double inv_t;
};

__device__ __forceinline__ float value_of(const float* p) { return *p; }
__device__ __forceinline__ float value_of(const uint16_t* p) { return __builtin_bit_cast(float, (uint32_t)*p << 16); }

// Logits in descending order, the lower id first among equals: larger keys come first.  NaN counts as -inf, -0 as 0.
__device__ __forceinline__ uint64_t key_of(float z, int id) {
    if (z != z) z = -INFINITY;
    const uint32_t b = __builtin_bit_cast(uint32_t, z + 0.0f);
    return (uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (uint32_t)~id;
}
__device__ __forceinline__ float value_of_key(uint64_t key) {
    const uint32_t b = (uint32_t)(key >> 32);
    return __builtin_bit_cast(float, b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ int id_of_key(uint64_t key) { return (int)~(uint32_t)key; }

// A workgroup a row; K more passes over the row for the alternatives.
template <typename T>
__global__ __launch_bounds__(kThreads) void logprob_row_kernel(LogprobArgs a) {
    __shared__ double sums[2][kThreads / kWave];
    __shared__ uint64_t keys[kThreads / kWave];
    const int row = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (a.n_rows && row >= a.n_rows[0]) return;
    const T* z = (const T*)a.logits + row * a.stride;
    auto best_below = [&](uint64_t bound) {
        uint64_t best = 0;
        for (int v = threadIdx.x; v < a.V; v += kThreads) {
            const uint64_t k = key_of(value_of(z + v), v);
            if (k < bound && k > best) best = k;
        }
        for (int o = 32; o > 0; o >>= 1) {
            const uint64_t other = (uint64_t)(uint32_t)__shfl_xor((int)(best >> 32), o, kWave) << 32 | (uint32_t)__shfl_xor((int)best, o, kWave);
            best = other > best ? other : best;
        }
        __syncthreads();
        if (lane == 0) keys[wave] = best;
        __syncthreads();
        for (int w = 0; w < kThreads / kWave; ++w) best = keys[w] > best ? keys[w] : best;
        return best;
    };
    const uint64_t first = best_below(~0ull);
    const float m = value_of_key(first);
    float s = 0.0f, e = 0.0f;
    for (int v = threadIdx.x; v < a.V; v += kThreads) {
        const float x = fmaxf((value_of(z + v) - m) * a.scale, -200.0f);  // (NaN, -inf: no weight)
        const float w = __builtin_amdgcn_exp2f(x);
        s += w;
        e = fmaf(w, x, e);
    }
    const double ws = wave_sum((double)s), we = wave_sum((double)e);
    if (lane == 0) { sums[0][wave] = ws; sums[1][wave] = we; }
    __syncthreads();
    double S = 0.0, E = 0.0;
    for (int w = 0; w < kThreads / kWave; ++w) { S += sums[0][w]; E += sums[1][w]; }
    const bool none = !(fabsf(m) < INFINITY);  // no finite logit, or one that is infinite
    const double log_s = none ? __builtin_nan("") : log(S);
    auto logprob = [&](float zv) { return (float)(((double)zv - (double)m) * a.inv_t - log_s); };
    if (threadIdx.x == 0 && a.entropy) a.entropy[row] = (float)(log_s - E / S * kLn2);
    for (int t = threadIdx.x; t < a.M; t += kThreads) {
        const int id = a.tokens[(size_t)row * a.M + t];
        float zv = id >= 0 && id < a.V ? value_of(z + id) : -INFINITY;
        if (zv != zv) zv = -INFINITY;
        a.logprobs[(size_t)row * a.M + t] = logprob(zv);
    }
    uint64_t key = first;
    for (int k = 0; k < a.K; ++k) {
        if (k) key = best_below(key);
        if (threadIdx.x == 0) {
            a.top_ids[(size_t)row * a.K + k] = id_of_key(key);
            a.top_logprobs[(size_t)row * a.K + k] = logprob(value_of_key(key));
        }
    }
}

int check(const fsr_logprob_params* p, const char* who) {
    if (!p) return fail(FSR_EINVAL, "%s: params is null", who);
    if (p->N_cap < 0 || p->V <= 0 || p->M < 0 || p->K < 0 || p->reserved != 0)
        return fail(FSR_EINVAL, "%s: N_cap=%d V=%d M=%d K=%d reserved=%d", who, p->N_cap, p->V, p->M, p->K, p->reserved);
    if (p->dtype != FSR_F32 && p->dtype != FSR_BF16) return fail(FSR_EUNSUP, "%s: dtype=%d", who, p->dtype);
    if (p->K > FSR_TOP_MAX) return fail(FSR_EUNSUP, "%s: K=%d alternatives (up to %d are built)", who, p->K, FSR_TOP_MAX);
    if (p->K > p->V) return fail(FSR_ESHAPE, "%s: K=%d of V=%d tokens", who, p->K, p->V);
    if (p->stride < p->V) return fail(FSR_ESHAPE, "%s: rows overlap (stride=%lld V=%d)", who, (long long)p->stride, p->V);
    if (!(p->temperature >= 1e-6) || !(p->temperature <= 1e6)) return fail(FSR_EINVAL, "%s: temperature=%g must be 1e-6 .. 1e6", who, p->temperature);
    if (p->N_cap > (1 << 22)) return fail(FSR_EUNSUP, "%s: N_cap=%d exceeds 2^22 rows", who, p->N_cap);
    return FSR_OK;
}

}  // namespace
}  // namespace fsr

using namespace fsr;

extern "C" int fsr_logprob_workspace_bytes(const fsr_logprob_params* p, size_t* out_bytes) {
    int rc = check(p, "fsr_logprob_workspace_bytes");
    if (rc != FSR_OK) return rc;
    if (!out_bytes) return fail(FSR_EINVAL, "fsr_logprob_workspace_bytes: out_bytes is null");
    *out_bytes = 256;
    return FSR_OK;
}

extern "C" int fsr_token_logprobs(const void* logits, const int32_t* n_rows, const int32_t* tokens, float* logprobs, float* entropy, int32_t* top_ids,
                                  float* top_logprobs, const fsr_logprob_params* p, void* workspace, size_t ws_bytes, void* stream) {
    const char* who = "fsr_token_logprobs";
    int rc = check(p, who);
    if (rc != FSR_OK) return rc;
    if (p->N_cap == 0) return FSR_OK;
    if (!logits || (p->M > 0 && (!tokens || !logprobs)) || (p->K > 0 && (!top_ids || !top_logprobs)))
        return fail(FSR_EINVAL, "%s: null pointer among logits/tokens/logprobs/top_ids/top_logprobs", who);
    if ((uintptr_t)logits & (p->dtype == FSR_F32 ? 3 : 1)) return fail(FSR_EINVAL, "%s: logits must be aligned to their elements", who);
    size_t need;
    fsr_logprob_workspace_bytes(p, &need);
    if (!workspace || ws_bytes < need) return fail(FSR_EWS, "%s: workspace %zu bytes, need %zu", who, ws_bytes, need);
    if ((uintptr_t)workspace & 255) return fail(FSR_EWS, "%s: workspace must be 256-byte aligned", who);
    LogprobArgs a{};
    a.logits = logits; a.n_rows = n_rows; a.tokens = tokens; a.logprobs = logprobs; a.entropy = entropy; a.top_ids = top_ids; a.top_logprobs = top_logprobs;
    a.stride = p->stride; a.N_cap = p->N_cap; a.V = p->V; a.M = p->M; a.K = p->K;
    a.scale = (float)(kLog2e / p->temperature);
    a.inv_t = 1.0 / p->temperature;
    if (p->dtype == FSR_F32) hipLaunchKernelGGL((logprob_row_kernel<float>), dim3(p->N_cap), dim3(kThreads), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL((logprob_row_kernel<uint16_t>), dim3(p->N_cap), dim3(kThreads), 0, (hipStream_t)stream, a);
    return check_launch(who);
}
