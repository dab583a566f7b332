// Newton-Schulz iteration X <- c0 X + (c1 G + c2 G G) X with G = X X^T on a batch of matrices, and the weight update by
// an orthogonalised momentum.  fp32 tiles of 32 x 32 through shared memory, one thread per 2 x 2 results.
#include <hip/hip_runtime.h>

#include <cmath>

#include "operator_types.h"

namespace marl {
namespace {

constexpr int kTile = 32, kDepth = 32;

// D = alpha A op(B) + beta C for matrices [M, K], [K, N] (or [N, K]: TRANSPOSED), dense, one batch member per blockIdx.z.
template <bool TRANSPOSED>
__global__ __launch_bounds__(256) void product_kernel(int M, int N, int K, const float *A, const float *B, const float *C, float *D,
                                                      float alpha, float beta)
{
    __shared__ float a[kTile][kDepth + 1], b[kTile][kDepth + 1];
    A += (size_t)blockIdx.z * M * K;
    B += (size_t)blockIdx.z * K * N;
    C += (size_t)blockIdx.z * M * N;
    D += (size_t)blockIdx.z * M * N;
    const int m0 = blockIdx.y * kTile, n0 = blockIdx.x * kTile;
    const int tr = threadIdx.x / 16, tc = threadIdx.x % 16;
    float acc[2][2] = {};
    for (int k0 = 0; k0 < K; k0 += kDepth) {
        for (int e = threadIdx.x; e < kTile * kDepth; e += 256) {
            const int r = e / kDepth, k = e % kDepth;
            a[r][k] = m0 + r < M && k0 + k < K ? A[(size_t)(m0 + r) * K + k0 + k] : 0.0f;
            if constexpr (TRANSPOSED) b[r][k] = n0 + r < N && k0 + k < K ? B[(size_t)(n0 + r) * K + k0 + k] : 0.0f;
            else b[k][r] = n0 + k < N && k0 + r < K ? B[(size_t)(k0 + r) * N + n0 + k] : 0.0f;
        }
        __syncthreads();
        for (int k = 0; k < kDepth; ++k)
            for (int i = 0; i < 2; ++i)
                for (int j = 0; j < 2; ++j) acc[i][j] = fmaf(a[tr + 16 * i][k], b[tc + 16 * j][k], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j) {
            const int m = m0 + tr + 16 * i, n = n0 + tc + 16 * j;
            if (m < M && n < N) D[(size_t)m * N + n] = alpha * acc[i][j] + (beta != 0.0f ? beta * C[(size_t)m * N + n] : 0.0f);
        }
}

struct UpdateArgs {
    int rows, cols;
    bool tall;                 // X is the transpose
    const void *weights, *grad;
    const float *momentum;
    void *weights_out;
    float *momentum_out;
    float beta;
    int nesterov;
    float keep, rate;          // weights_out = keep weights - rate X
    float *X;
    double *norm;              // [L] sum of squares
};

// X = the matrix (or its momentum) in fp32, and the sum of its squares: one workgroup per matrix.
template <typename E>
__global__ __launch_bounds__(1024) void start_kernel(UpdateArgs p)
{
    __shared__ double part[1024 / kWave];
    const size_t n = (size_t)p.rows * p.cols, base = blockIdx.x * n;
    double sum = 0.0;
    for (size_t k = threadIdx.x; k < n; k += 1024) {
        float u = to_f32(static_cast<const E *>(p.grad)[base + k]);
        if (p.momentum) {
            const float m = fmaf(p.beta, p.momentum[base + k], u);
            p.momentum_out[base + k] = m;
            u = p.nesterov ? fmaf(p.beta, m, u) : m;
        }
        const size_t r = k / p.cols, c = k % p.cols;
        p.X[base + (p.tall ? c * p.rows + r : k)] = u;
        sum += (double)u * u;
    }
    for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0;
        for (int w = 0; w < 1024 / kWave; ++w) sum += part[w];
        p.norm[blockIdx.x] = sum;
    }
}

__global__ __launch_bounds__(256) void scale_kernel(float *X, size_t n, const double *norm, float eps)
{
    const size_t k = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (k >= n) return;
    X[blockIdx.y * n + k] = (float)(X[blockIdx.y * n + k] / fmax(sqrt(norm[blockIdx.y]), (double)eps));
}

template <typename E>
__global__ __launch_bounds__(256) void finish_kernel(UpdateArgs p)
{
    const size_t n = (size_t)p.rows * p.cols, k = (size_t)blockIdx.x * 256 + threadIdx.x, base = blockIdx.y * n;
    if (k >= n) return;
    const size_t r = k / p.cols, c = k % p.cols;
    const float x = p.X[base + (p.tall ? c * p.rows + r : k)];
    E *out = static_cast<E *>(p.weights_out) + base + k;
    *out = from_f32<E>(p.weights ? p.keep * to_f32(static_cast<const E *>(p.weights)[base + k]) - p.rate * x : x);
}

bool sizes_ok(int L, int rows, int cols) { return L >= 0 && L <= 65535 && rows >= 1 && cols >= 1 && rows <= 32768 && cols <= 32768; }

size_t up(size_t n) { return (n + 255) / 256 * 256; }

struct Layout {
    size_t x[2], g, p, norm, bytes;
};

Layout layout_of(int L, int rows, int cols)
{
    const size_t s = rows < cols ? rows : cols, n = (size_t)rows * cols;
    Layout l;
    size_t at = 0;
    for (size_t &x : l.x) { x = at; at += up(L * n * sizeof(float)); }
    l.g = at; at += up(L * s * s * sizeof(float));
    l.p = at; at += up(L * s * s * sizeof(float));
    l.norm = at; at += up(L * sizeof(double));
    l.bytes = at;
    return l;
}

int newton_schulz(int dtype, int L, UpdateArgs p, char *workspace, int steps, const float *coef, float eps, hipStream_t stream)
{
    const Layout l = layout_of(L, p.rows, p.cols);
    const int s = p.rows < p.cols ? p.rows : p.cols, len = p.rows < p.cols ? p.cols : p.rows;
    const size_t n = (size_t)p.rows * p.cols;
    float *X[2] = {reinterpret_cast<float *>(workspace + l.x[0]), reinterpret_cast<float *>(workspace + l.x[1])};
    float *G = reinterpret_cast<float *>(workspace + l.g), *P = reinterpret_cast<float *>(workspace + l.p);
    p.tall = p.rows > p.cols;
    p.X = X[0];
    p.norm = reinterpret_cast<double *>(workspace + l.norm);
    const dim3 each((unsigned)((n + 255) / 256), (unsigned)L);
    const unsigned ts = (unsigned)((s + kTile - 1) / kTile), tl = (unsigned)((len + kTile - 1) / kTile);
    with_dtype(dtype, [&](auto e) {
        hipLaunchKernelGGL((start_kernel<decltype(e)>), dim3((unsigned)L), dim3(1024), 0, stream, p);
        return 0;
    });
    hipLaunchKernelGGL(scale_kernel, each, dim3(256), 0, stream, X[0], n, p.norm, eps);
    for (int k = 0; k < steps; ++k) {
        hipLaunchKernelGGL(product_kernel<true>, dim3(ts, ts, L), dim3(256), 0, stream, s, s, len, X[0], X[0], G, G, 1.0f, 0.0f);
        hipLaunchKernelGGL(product_kernel<false>, dim3(ts, ts, L), dim3(256), 0, stream, s, s, s, G, G, G, P, coef[2], coef[1]);
        hipLaunchKernelGGL(product_kernel<false>, dim3(tl, ts, L), dim3(256), 0, stream, s, len, s, P, X[0], X[0], X[1], 1.0f, coef[0]);
        float *t = X[0]; X[0] = X[1]; X[1] = t;
    }
    p.X = X[0];
    return with_dtype(dtype, [&](auto e) {
        hipLaunchKernelGGL((finish_kernel<decltype(e)>), each, dim3(256), 0, stream, p);
        return launched("orthogonalised update");
    });
}

int check(int dtype, int L, int rows, int cols, const void *workspace, size_t workspace_bytes, int steps, const float *coef, float eps)
{
    if (!known_dtype(dtype)) return MARL_ERR_BAD_DTYPE;
    if (!sizes_ok(L, rows, cols)) return MARL_ERR_BAD_DIM;
    if (!coef) return MARL_ERR_NULL;
    for (int k = 0; k < 3; ++k)
        if (!std::isfinite(coef[k])) return MARL_ERR_BAD_ARG;
    if (steps < 0 || steps > 64 || !std::isfinite(eps) || !(eps > 0.0f)) return MARL_ERR_BAD_ARG;
    if (workspace_bytes < layout_of(L, rows, cols).bytes) return MARL_ERR_BAD_DIM;
    if (!workspace && workspace_bytes) return MARL_ERR_NULL;
    return aligned_to(workspace, 256) ? MARL_OK : MARL_ERR_BAD_ARG;
}

}  // namespace
}  // namespace marl

using namespace marl;

extern "C" {

int marl_muon_workspace_bytes(int32_t dtype, int32_t L, int32_t rows, int32_t cols, size_t *bytes)
{
    if (!bytes) return MARL_ERR_NULL;
    if (!known_dtype(dtype)) return MARL_ERR_BAD_DTYPE;
    if (!sizes_ok(L, rows, cols)) return MARL_ERR_BAD_DIM;
    *bytes = layout_of(L, rows, cols).bytes;
    return MARL_OK;
}

int marl_orthogonalize(int32_t dtype, int32_t L, int32_t rows, int32_t cols, const void *matrix, void *out,
                       void *workspace, size_t workspace_bytes, int32_t steps, const float *coefficients, float eps,
                       void *hip_stream)
{
    const int rc = check(dtype, L, rows, cols, workspace, workspace_bytes, steps, coefficients, eps);
    if (rc) return rc;
    if (L == 0) return MARL_OK;
    if (!matrix || !out) return MARL_ERR_NULL;
    UpdateArgs p{};
    p.rows = rows; p.cols = cols; p.grad = matrix; p.weights_out = out;
    return newton_schulz(dtype, L, p, static_cast<char *>(workspace), steps, coefficients, eps, static_cast<hipStream_t>(hip_stream));
}

int marl_muon_step(int32_t dtype, int32_t L, int32_t rows, int32_t cols, const void *weights, const void *grad,
                   const float *momentum, void *weights_out, float *momentum_out, void *workspace,
                   size_t workspace_bytes, float lr, float beta, int32_t nesterov, float weight_decay, float scale,
                   int32_t steps, const float *coefficients, float eps, void *hip_stream)
{
    const int rc = check(dtype, L, rows, cols, workspace, workspace_bytes, steps, coefficients, eps);
    if (rc) return rc;
    if (!std::isfinite(lr) || !std::isfinite(beta) || !std::isfinite(weight_decay) || !std::isfinite(scale)) return MARL_ERR_BAD_ARG;
    if (L == 0) return MARL_OK;
    if (!weights || !grad || !momentum || !weights_out || !momentum_out) return MARL_ERR_NULL;
    UpdateArgs p{};
    p.rows = rows; p.cols = cols; p.weights = weights; p.grad = grad; p.momentum = momentum;
    p.weights_out = weights_out; p.momentum_out = momentum_out; p.beta = beta; p.nesterov = nesterov;
    p.keep = (float)(1.0 - (double)lr * weight_decay);
    p.rate = (float)((double)lr * scale);
    return newton_schulz(dtype, L, p, static_cast<char *>(workspace), steps, coefficients, eps, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
