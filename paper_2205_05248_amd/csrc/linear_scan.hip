// Gated linear recurrence: h[t] = a[t] h[t-1] + beta[t] sigmoid(i[t]) x[t], its backward pass and its form for one step.
// One thread walks one channel of one sequence.
#include <hip/hip_runtime.h>

#include <cmath>

#include "device_math.h"
#include "operator_types.h"

namespace marl {
namespace {

constexpr int kKeep = 16;              // steps between the states that the backward pass starts from

struct ScanArgs {
    int B, T, C;
    const void *x, *r, *i;
    int64_t ld_x, ld_r, ld_i;
    const float *lam;
    float decay;
    const uint8_t *reset, *filled;
    const float *h_first;
    void *y;
    int64_t ld_y;
    float *h_last;
    float *states;                     // [B, ceil(T / kKeep), C] state before each kKeep-th step
    // backward pass
    const void *grad_y;
    int64_t ld_gy;
    const float *grad_h_last;
    void *grad_x, *grad_r, *grad_i;
    int64_t ld_gx, ld_gr, ld_gi;
    float *lam_part;                   // [B, C]
    float *grad_lam, *grad_h_first;
};

__device__ __forceinline__ float rate_of(float lam, float decay)
{
    return decay * (lam > 20.0f ? lam : log1pf(expf(lam)));
}

// sigmoid(v) and its complement, each to fp32 accuracy at both ends.
struct Sigmoid { float s, c; };
__device__ __forceinline__ Sigmoid sigmoid2(float v)
{
    const float e = fminf(__builtin_amdgcn_exp2f(-kLog2e * v), 1e37f);
    const float s = __builtin_amdgcn_rcpf(1.0f + e);
    return {s, e * s};
}

// 1 - exp(y) for y <= 0.  Near 0 the difference would cancel: there the series, whose next term is below 2^-25.
__device__ __forceinline__ float one_minus_exp(float y, float exp_y)
{
    float p = fmaf(y, 1.0f / 7.0f, 1.0f);
    p = fmaf(y * (1.0f / 6.0f), p, 1.0f);
    p = fmaf(y * 0.2f, p, 1.0f);
    p = fmaf(y * 0.25f, p, 1.0f);
    p = fmaf(y * (1.0f / 3.0f), p, 1.0f);
    p = fmaf(y * 0.5f, p, 1.0f);
    return y > -0.35f ? -y * p : 1.0f - exp_y;
}

struct Gates { Sigmoid sr, si; float a, inv_beta, beta; };
__device__ __forceinline__ Gates gates_of(float r, float i, float rate)
{
    Gates g;
    g.sr = sigmoid2(r);
    g.si = sigmoid2(i);
    const float L = -rate * g.sr.s;
    g.a = __builtin_amdgcn_exp2f(kLog2e * L);
    const float om = one_minus_exp(2.0f * L, g.a * g.a);
    g.inv_beta = __builtin_amdgcn_rsqf(fmaxf(om, 1e-30f));     // a gate that is shut has om = 0: beta 0, and no infinity
    g.beta = om * g.inv_beta;
    return g;
}

// What one step does to the state: h <- a h + u.  kind 0: padding, 1: start of a sequence, 2: ordinary.
__device__ __forceinline__ int step_kind(const ScanArgs &p, int64_t row)
{
    if (p.filled && !p.filled[row]) return 0;
    return p.reset && p.reset[row] ? 1 : 2;
}

template <typename E>
__global__ __launch_bounds__(256) void scan_kernel(ScanArgs p)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (int64_t)p.B * p.C) return;
    const int b = (int)(id / p.C), c = (int)(id % p.C);
    const E *x = static_cast<const E *>(p.x), *r = static_cast<const E *>(p.r), *i = static_cast<const E *>(p.i);
    const float rate = rate_of(p.lam[c], p.decay);
    const int chunks = (p.T + kKeep - 1) / kKeep;
    float h = p.h_first ? p.h_first[id] : 0.0f;
    for (int t = 0; t < p.T; ++t) {
        const int64_t row = (int64_t)b * p.T + t;
        if (t % kKeep == 0) p.states[((int64_t)b * chunks + t / kKeep) * p.C + c] = h;
        const int kind = step_kind(p, row);
        if (kind) {
            const Gates g = gates_of(to_f32(r[row * p.ld_r + c]), to_f32(i[row * p.ld_i + c]), rate);
            const float in = g.si.s * to_f32(x[row * p.ld_x + c]);
            h = kind == 1 ? in : fmaf(g.a, h, g.beta * in);
        }
        static_cast<E *>(p.y)[row * p.ld_y + c] = from_f32<E>(kind ? h : 0.0f);
    }
    if (p.h_last) p.h_last[id] = h;
}

template <typename E>
__global__ __launch_bounds__(256) void scan_grad_kernel(ScanArgs p)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (int64_t)p.B * p.C) return;
    const int b = (int)(id / p.C), c = (int)(id % p.C);
    const E *x = static_cast<const E *>(p.x), *r = static_cast<const E *>(p.r), *i = static_cast<const E *>(p.i);
    const E *gy = static_cast<const E *>(p.grad_y);
    const float rate = rate_of(p.lam[c], p.decay);
    const int chunks = (p.T + kKeep - 1) / kKeep;
    float dh = p.grad_h_last ? p.grad_h_last[id] : 0.0f;       // dL/dh after the step in hand
    float sum = 0.0f;
    for (int k = chunks - 1; k >= 0; --k) {
        float before[kKeep];
        float h = p.states[((int64_t)b * chunks + k) * p.C + c];
        const int t0 = k * kKeep, n = min(kKeep, p.T - t0);
#pragma unroll
        for (int j = 0; j < kKeep; ++j) {
            before[j] = h;
            if (j >= n) continue;
            const int64_t row = (int64_t)b * p.T + t0 + j;
            const int kind = step_kind(p, row);
            if (!kind) continue;
            const Gates g = gates_of(to_f32(r[row * p.ld_r + c]), to_f32(i[row * p.ld_i + c]), rate);
            const float in = g.si.s * to_f32(x[row * p.ld_x + c]);
            h = kind == 1 ? in : fmaf(g.a, h, g.beta * in);
        }
#pragma unroll
        for (int j = kKeep - 1; j >= 0; --j) {
            if (j >= n) continue;
            const int64_t row = (int64_t)b * p.T + t0 + j;
            const int kind = step_kind(p, row);
            float dx = 0.0f, dr = 0.0f, di = 0.0f;
            if (kind) {
                const float xv = to_f32(x[row * p.ld_x + c]);
                const Gates g = gates_of(to_f32(r[row * p.ld_r + c]), to_f32(i[row * p.ld_i + c]), rate);
                dh += to_f32(gy[row * p.ld_gy + c]);
                const float du = kind == 1 ? dh : dh * g.beta;
                dx = du * g.si.s;
                di = du * xv * g.si.s * g.si.c;
                if (kind == 2) {
                    const float dL = g.a * dh * (before[j] - g.si.s * xv * g.a * g.inv_beta);
                    dr = -rate * g.sr.s * g.sr.c * dL;
                    sum -= g.sr.s * dL;
                    dh *= g.a;
                } else {
                    dh = 0.0f;
                }
            }
            static_cast<E *>(p.grad_x)[row * p.ld_gx + c] = from_f32<E>(dx);
            static_cast<E *>(p.grad_r)[row * p.ld_gr + c] = from_f32<E>(dr);
            static_cast<E *>(p.grad_i)[row * p.ld_gi + c] = from_f32<E>(di);
        }
    }
    if (p.grad_h_first) p.grad_h_first[id] = dh;
    p.lam_part[id] = sum;
}

// grad_lam[c] = decay sigmoid(lam[c]) * sum of the sequences' parts, in order.
__global__ __launch_bounds__(256) void scan_lam_kernel(ScanArgs p)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= p.C) return;
    float sum = 0.0f;
    for (int b = 0; b < p.B; ++b) sum += p.lam_part[(int64_t)b * p.C + c];
    p.grad_lam[c] = sum * p.decay * sigmoid2(p.lam[c]).s;
}

struct StepArgs {
    int n, C, slots;
    const void *x, *r, *i;
    int64_t ld_x, ld_r, ld_i;
    const float *lam;
    float decay;
    const int32_t *slot;
    const uint8_t *reset;
    const float *h_in;
    float *h_out;
    void *y;
    int64_t ld_y;
};

template <typename E>
__global__ __launch_bounds__(256) void step_kernel(StepArgs p)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (int64_t)p.n * p.C) return;
    const int64_t row = id / p.C;
    const int c = (int)(id % p.C);
    const int64_t at = (int64_t)(p.slot ? min(max(p.slot[row], 0), p.slots - 1) : (int)row) * p.C + c;
    const Gates g = gates_of(to_f32(static_cast<const E *>(p.r)[row * p.ld_r + c]),
                             to_f32(static_cast<const E *>(p.i)[row * p.ld_i + c]), rate_of(p.lam[c], p.decay));
    const float in = g.si.s * to_f32(static_cast<const E *>(p.x)[row * p.ld_x + c]);
    const float h = p.reset && p.reset[row] ? in : fmaf(g.a, p.h_in[at], g.beta * in);
    p.h_out[at] = h;
    static_cast<E *>(p.y)[row * p.ld_y + c] = from_f32<E>(h);
}

size_t scan_states(int B, int T, int C) { return (size_t)B * ((T + kKeep - 1) / kKeep) * C; }

bool scan_sizes_ok(int B, int T, int C)
{
    return B >= 0 && T >= 0 && C >= 0 && C < (1 << 24) && (int64_t)B * T < ((int64_t)1 << 30);
}

size_t scan_workspace(int B, int T, int C)
{
    const size_t bytes = (scan_states(B, T, C) + (size_t)B * C) * sizeof(float);
    return (bytes + 255) / 256 * 256;
}

bool positive(float v) { return std::isfinite(v) && v > 0.0f; }

// Checks that the forward and the backward call have in common.
int scan_check(int dtype, int B, int T, int C, float decay, const void *workspace, size_t workspace_bytes)
{
    if (!known_dtype(dtype)) return MARL_ERR_BAD_DTYPE;
    if (!scan_sizes_ok(B, T, C)) return MARL_ERR_BAD_DIM;
    if (!positive(decay)) return MARL_ERR_BAD_ARG;
    if (workspace_bytes < scan_workspace(B, T, C)) return MARL_ERR_BAD_DIM;
    if (!workspace && workspace_bytes) return MARL_ERR_NULL;
    return aligned_to(workspace, 256) ? MARL_OK : MARL_ERR_BAD_ARG;
}

unsigned blocks_of(int64_t n) { return (unsigned)((n + 255) / 256); }

}  // namespace
}  // namespace marl

using namespace marl;

extern "C" {

int marl_linear_scan_workspace_bytes(int32_t dtype, int32_t B, int32_t T, int32_t C, size_t *bytes)
{
    if (!bytes) return MARL_ERR_NULL;
    if (!known_dtype(dtype)) return MARL_ERR_BAD_DTYPE;
    if (!scan_sizes_ok(B, T, C)) return MARL_ERR_BAD_DIM;
    *bytes = scan_workspace(B, T, C);
    return MARL_OK;
}

int marl_linear_scan(int32_t dtype, int32_t B, int32_t T, int32_t C, const void *x, int64_t ld_x, const void *r,
                     int64_t ld_r, const void *i, int64_t ld_i, const float *lam, float decay, const uint8_t *reset,
                     const uint8_t *filled, const float *h_first, void *y, int64_t ld_y, float *h_last,
                     void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const int rc = scan_check(dtype, B, T, C, decay, workspace, workspace_bytes);
    if (rc) return rc;
    if (B == 0 || C == 0) return MARL_OK;
    if (!lam || (T > 0 && (!x || !r || !i || !y))) return MARL_ERR_NULL;
    if (ld_x < C || ld_r < C || ld_i < C || ld_y < C) return MARL_ERR_BAD_DIM;
    if (T > 0 && (y == x || y == r || y == i)) return MARL_ERR_BAD_ARG;
    ScanArgs p{};
    p.B = B; p.T = T; p.C = C;
    p.x = x; p.r = r; p.i = i; p.ld_x = ld_x; p.ld_r = ld_r; p.ld_i = ld_i;
    p.lam = lam; p.decay = decay; p.reset = reset; p.filled = filled; p.h_first = h_first;
    p.y = y; p.ld_y = ld_y; p.h_last = h_last; p.states = static_cast<float *>(workspace);
    return with_dtype(dtype, [&](auto e) {
        hipLaunchKernelGGL((scan_kernel<decltype(e)>), dim3(blocks_of((int64_t)B * C)), dim3(256), 0, static_cast<hipStream_t>(hip_stream), p);
        return launched("linear scan");
    });
}

int marl_linear_scan_grad(int32_t dtype, int32_t B, int32_t T, int32_t C, const void *x, int64_t ld_x, const void *r,
                          int64_t ld_r, const void *i, int64_t ld_i, const float *lam, float decay,
                          const uint8_t *reset, const uint8_t *filled, const void *grad_y, int64_t ld_gy,
                          const float *grad_h_last, void *workspace, size_t workspace_bytes, void *grad_x,
                          int64_t ld_gx, void *grad_r, int64_t ld_gr, void *grad_i, int64_t ld_gi, float *grad_lam,
                          float *grad_h_first, void *hip_stream)
{
    const int rc = scan_check(dtype, B, T, C, decay, workspace, workspace_bytes);
    if (rc) return rc;
    if (C == 0) return MARL_OK;
    if (!lam || !grad_lam || (B > 0 && T > 0 && (!x || !r || !i || !grad_y || !grad_x || !grad_r || !grad_i))) return MARL_ERR_NULL;
    if (ld_x < C || ld_r < C || ld_i < C || ld_gy < C || ld_gx < C || ld_gr < C || ld_gi < C) return MARL_ERR_BAD_DIM;
    const void *in[4] = {x, r, i, grad_y}, *out[3] = {grad_x, grad_r, grad_i};
    for (int k = 0; k < 3; ++k) {
        for (const void *v : in)
            if (v && out[k] == v) return MARL_ERR_BAD_ARG;
        if (out[k] && out[k] == out[(k + 1) % 3]) return MARL_ERR_BAD_ARG;
    }
    ScanArgs p{};
    p.B = B; p.T = T; p.C = C;
    p.x = x; p.r = r; p.i = i; p.ld_x = ld_x; p.ld_r = ld_r; p.ld_i = ld_i;
    p.lam = lam; p.decay = decay; p.reset = reset; p.filled = filled;
    p.states = static_cast<float *>(workspace);
    p.grad_y = grad_y; p.ld_gy = ld_gy; p.grad_h_last = grad_h_last;
    p.grad_x = grad_x; p.grad_r = grad_r; p.grad_i = grad_i; p.ld_gx = ld_gx; p.ld_gr = ld_gr; p.ld_gi = ld_gi;
    p.lam_part = p.states + scan_states(B, T, C);
    p.grad_lam = grad_lam; p.grad_h_first = grad_h_first;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (B > 0) {
        const int status = with_dtype(dtype, [&](auto e) {
            hipLaunchKernelGGL((scan_grad_kernel<decltype(e)>), dim3(blocks_of((int64_t)B * C)), dim3(256), 0, stream, p);
            return launched("linear scan gradient");
        });
        if (status) return status;
    }
    hipLaunchKernelGGL(scan_lam_kernel, dim3(blocks_of(C)), dim3(256), 0, stream, p);
    return launched("linear scan gradient");
}

int marl_linear_step(int32_t dtype, int32_t n, int32_t C, const void *x, int64_t ld_x, const void *r, int64_t ld_r,
                     const void *i, int64_t ld_i, const float *lam, float decay, const int32_t *slot, int32_t slots,
                     const uint8_t *reset, const float *h_in, float *h_out, void *y, int64_t ld_y, void *hip_stream)
{
    if (!known_dtype(dtype)) return MARL_ERR_BAD_DTYPE;
    if (n < 0 || C < 0 || C >= (1 << 24) || slots < 1 || (!slot && n > slots) || (int64_t)n * C >= ((int64_t)1 << 38)) return MARL_ERR_BAD_DIM;
    if (!positive(decay)) return MARL_ERR_BAD_ARG;
    if (n == 0 || C == 0) return MARL_OK;
    if (!x || !r || !i || !lam || !h_in || !h_out || !y) return MARL_ERR_NULL;
    if (ld_x < C || ld_r < C || ld_i < C || ld_y < C) return MARL_ERR_BAD_DIM;
    if (y == x || y == r || y == i) return MARL_ERR_BAD_ARG;
    const StepArgs p{n, C, slots, x, r, i, ld_x, ld_r, ld_i, lam, decay, slot, reset, h_in, h_out, y, ld_y};
    return with_dtype(dtype, [&](auto e) {
        hipLaunchKernelGGL((step_kernel<decltype(e)>), dim3(blocks_of((int64_t)n * C)), dim3(256), 0, static_cast<hipStream_t>(hip_stream), p);
        return launched("linear step");
    });
}

}  // extern "C"
