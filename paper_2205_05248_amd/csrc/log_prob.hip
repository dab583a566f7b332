// Log probability of given tokens, entropy and most likely alternatives of rows of logits, and the logits' gradient.
// One workgroup per row: one pass with a running maximum m, sum s = sum e^(z-m) and moment w = sum e^(z-m) (z-m), from which
// log_sum = m + log s and entropy = log s - w / s.
#include <hip/hip_runtime.h>

#include <cmath>

#include "device_math.h"
#include "operator_types.h"

namespace marl {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTop = 64;
constexpr float kInf = __builtin_inff();

struct LogProbArgs {
    int R, V, K;
    const void *logits;
    int64_t ld;
    const int32_t *token;
    const uint8_t *avail;
    int64_t ld_avail;
    float scale;
    float *logp, *entropy, *log_sum;
    int32_t *top_id;
    float *top_logp;
    // gradient
    const float *in_log_sum, *in_entropy, *grad_logp, *grad_entropy;
    void *grad_logits;
    int64_t ld_grad;
};

// Running statistics of a set of z; m = -inf is the empty set.
struct Stats {
    float m, s, w;
};

// w of a set moved from maximum m to M >= m:  sum e^(z-M) (z-M) = e^(m-M) (w + (m-M) s).  Distances end at kFar, where
// e^ is 0 in fp32: the distance of a type's lowest value would make the product 0 * infinity.
constexpr float kFar = -200.0f;

// The lowest finite value stays finite under a scale above one.
__device__ __forceinline__ float scaled(float scale, float logit) { return fmaxf(scale * logit, -3.4028235e38f); }

__device__ __forceinline__ Stats join(Stats a, Stats b)
{
    const float M = fmaxf(a.m, b.m);
    if (!(M > -kInf)) return {-kInf, a.s + b.s, 0.0f};          // (a NaN stays in s)
    const float da = fmaxf(a.m - M, kFar), db = fmaxf(b.m - M, kFar);
    const float ea = a.m > -kInf ? __expf(da) : 0.0f, eb = b.m > -kInf ? __expf(db) : 0.0f;
    return {M, a.s * ea + b.s * eb, (a.m > -kInf ? ea * (a.w + da * a.s) : 0.0f) + (b.m > -kInf ? eb * (b.w + db * b.s) : 0.0f)};
}

template <typename E>
__global__ __launch_bounds__(kThreads) void log_prob_kernel(LogProbArgs p)
{
    __shared__ Stats part[kThreads / kWave];
    __shared__ float best_v[kThreads / kWave];
    __shared__ int best_j[kThreads / kWave];
    const int64_t row = blockIdx.x;
    const E *l = static_cast<const E *>(p.logits) + row * p.ld;
    const uint8_t *av = p.avail ? p.avail + row * p.ld_avail : nullptr;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    Stats st{-kInf, 0.0f, 0.0f};
    for (int j = threadIdx.x; j < p.V; j += kThreads) {
        if (av && !av[j]) continue;
        const float v = to_f32(l[j]);
        if (v == -kInf) continue;
        st = join(st, {scaled(p.scale, v), 1.0f, 0.0f});
        if (!(v < kInf)) st.s = __builtin_nanf("");             // NaN or +infinity: the row's values are NaN
    }
    for (int d = 1; d < kWave; d *= 2) st = join(st, {__shfl_xor(st.m, d), __shfl_xor(st.s, d), __shfl_xor(st.w, d)});
    if (lane == 0) part[wave] = st;
    __syncthreads();
    st = part[0];
    for (int w = 1; w < kThreads / kWave; ++w) st = join(st, part[w]);
    const bool none = st.s == 0.0f;
    const float log_s = logf(st.s);
    if (threadIdx.x == 0) {
        if (p.log_sum) p.log_sum[row] = none ? -kInf : st.m + log_s;
        if (p.entropy) p.entropy[row] = none ? 0.0f : log_s - st.w / st.s;
        if (p.logp) {
            const int tok = p.token ? p.token[row] : -1;
            float lp = 0.0f;
            if (!none && tok >= 0 && tok < p.V) {
                const float v = to_f32(l[tok]);
                lp = (av && !av[tok]) || v == -kInf ? -kInf : (scaled(p.scale, v) - st.m) - log_s;
            }
            p.logp[row] = lp;
        }
    }
    // the K largest, one after the other: the largest among those that come after the last one in (value, index) order
    float last_v = kInf;
    int last_j = -1;
    for (int k = 0; k < p.K; ++k) {
        float v = -kInf;
        int at = -1;
        for (int j = threadIdx.x; j < p.V; j += kThreads) {
            if (av && !av[j]) continue;
            const float x = to_f32(l[j]);
            if ((x < last_v || (x == last_v && j > last_j)) && x > v) { v = x; at = j; }
        }
        for (int d = 1; d < kWave; d *= 2) {
            const float ov = __shfl_xor(v, d);
            const int oj = __shfl_xor(at, d);
            if (oj >= 0 && (at < 0 || ov > v || (ov == v && oj < at))) { v = ov; at = oj; }
        }
        __syncthreads();
        if (lane == 0) { best_v[wave] = v; best_j[wave] = at; }
        __syncthreads();
        v = -kInf;
        at = -1;
        for (int w = 0; w < kThreads / kWave; ++w)
            if (best_j[w] >= 0 && (at < 0 || best_v[w] > v || (best_v[w] == v && best_j[w] < at))) { v = best_v[w]; at = best_j[w]; }
        if (threadIdx.x == 0) {
            p.top_id[row * p.K + k] = at;
            p.top_logp[row * p.K + k] = at < 0 ? -kInf : (scaled(p.scale, v) - st.m) - log_s;
        }
        if (at < 0) { last_v = -kInf; last_j = p.V; }
        else { last_v = v; last_j = at; }
    }
}

template <typename E>
__global__ __launch_bounds__(kThreads) void log_prob_grad_kernel(LogProbArgs p)
{
    const int64_t row = blockIdx.x;
    const E *l = static_cast<const E *>(p.logits) + row * p.ld;
    const uint8_t *av = p.avail ? p.avail + row * p.ld_avail : nullptr;
    E *out = static_cast<E *>(p.grad_logits) + row * p.ld_grad;
    const float log_sum = p.in_log_sum[row];
    const bool none = log_sum == -kInf;
    const int tok = p.grad_logp ? p.token[row] : -1;
    const bool has = !none && tok >= 0 && tok < p.V && !(av && !av[tok]) && to_f32(l[tok]) != -kInf;
    const float g_logp = has ? p.grad_logp[row] : 0.0f;
    const float g_ent = p.grad_entropy ? p.grad_entropy[row] : 0.0f, ent = p.grad_entropy ? p.in_entropy[row] : 0.0f;
    __syncthreads();                                            // the token's logit is read before it may be overwritten
    for (int j = threadIdx.x; j < p.V; j += kThreads) {
        float g = 0.0f;
        if (!none && !(av && !av[j])) {
            const float v = to_f32(l[j]);
            if (v != -kInf) {
                // p as the square of its root, which the hardware exponential does not flush where p is subnormal
                const float lp = fmaxf(scaled(p.scale, v) - log_sum, kFar), root = __builtin_amdgcn_exp2f(0.5f * kLog2e * lp);
                g = p.scale * ((has && j == tok ? g_logp : 0.0f) - root * (root * (g_logp + g_ent * (lp + ent))));
            }
        }
        out[j] = from_f32<E>(g);
    }
}

int log_prob_check(int dtype, int R, int V, const void *logits, int64_t ld, const uint8_t *avail, int64_t ld_avail, float scale)
{
    if (!known_dtype(dtype)) return MARL_ERR_BAD_DTYPE;
    if (R < 0 || V < 1 || V >= (1 << 30) || ld < V) return MARL_ERR_BAD_DIM;
    if (avail && ld_avail != 0 && ld_avail < V) return MARL_ERR_BAD_DIM;
    if (!std::isfinite(scale) || !(scale > 0.0f)) return MARL_ERR_BAD_ARG;
    return !logits && R > 0 ? MARL_ERR_NULL : MARL_OK;
}

size_t log_prob_workspace(int, int, int) { return 0; }

}  // namespace
}  // namespace marl

using namespace marl;

extern "C" {

int marl_log_prob_workspace_bytes(int32_t R, int32_t V, int32_t K, size_t *bytes)
{
    if (!bytes) return MARL_ERR_NULL;
    if (R < 0 || V < 1 || V >= (1 << 30) || K < 0 || K > kMaxTop) return MARL_ERR_BAD_DIM;
    *bytes = log_prob_workspace(R, V, K);
    return MARL_OK;
}

int marl_log_prob(int32_t dtype, int32_t R, int32_t V, const void *logits, int64_t ld, const int32_t *token,
                  const uint8_t *avail, int64_t ld_avail, float scale, float *logp, float *entropy, float *log_sum,
                  int32_t K, int32_t *top_id, float *top_logp, void *workspace, size_t workspace_bytes,
                  void *hip_stream)
{
    const int rc = log_prob_check(dtype, R, V, logits, ld, avail, ld_avail, scale);
    if (rc) return rc;
    if (K < 0 || K > kMaxTop || workspace_bytes < log_prob_workspace(R, V, K)) return MARL_ERR_BAD_DIM;
    if (R == 0) return MARL_OK;
    if ((logp && !token) || (K > 0 && (!top_id || !top_logp)) || (workspace_bytes && !workspace)) return MARL_ERR_NULL;
    if (!aligned_to(workspace, 256)) return MARL_ERR_BAD_ARG;
    LogProbArgs p{};
    p.R = R; p.V = V; p.K = K;
    p.logits = logits; p.ld = ld; p.token = token; p.avail = avail; p.ld_avail = ld_avail; p.scale = scale;
    p.logp = logp; p.entropy = entropy; p.log_sum = log_sum; p.top_id = top_id; p.top_logp = top_logp;
    return with_dtype(dtype, [&](auto e) {
        hipLaunchKernelGGL((log_prob_kernel<decltype(e)>), dim3((unsigned)R), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), p);
        return launched("log prob");
    });
}

int marl_log_prob_grad(int32_t dtype, int32_t R, int32_t V, const void *logits, int64_t ld, const int32_t *token,
                       const uint8_t *avail, int64_t ld_avail, float scale, const float *log_sum,
                       const float *entropy, const float *grad_logp, const float *grad_entropy, void *grad_logits,
                       int64_t ld_grad, void *hip_stream)
{
    const int rc = log_prob_check(dtype, R, V, logits, ld, avail, ld_avail, scale);
    if (rc) return rc;
    if (ld_grad < V) return MARL_ERR_BAD_DIM;
    if (grad_logits && grad_logits == logits && ld_grad != ld) return MARL_ERR_BAD_ARG;
    if (R == 0) return MARL_OK;
    if (!log_sum || !grad_logits || (grad_logp && !token) || (grad_entropy && !entropy)) return MARL_ERR_NULL;
    LogProbArgs p{};
    p.R = R; p.V = V;
    p.logits = logits; p.ld = ld; p.token = token; p.avail = avail; p.ld_avail = ld_avail; p.scale = scale;
    p.in_log_sum = log_sum; p.in_entropy = entropy; p.grad_logp = grad_logp; p.grad_entropy = grad_entropy;
    p.grad_logits = grad_logits; p.ld_grad = ld_grad;
    return with_dtype(dtype, [&](auto e) {
        hipLaunchKernelGGL((log_prob_grad_kernel<decltype(e)>), dim3((unsigned)R), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), p);
        return launched("log prob gradient");
    });
}

}  // extern "C"
