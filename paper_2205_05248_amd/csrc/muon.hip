// Newton-Schulz iteration X <- c0 X + (c1 G + c2 G G) X with G = X X^T on a batch of matrices, and the weight update by
// an orthogonalised momentum.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "muon_small.h"

namespace marl {
namespace {

struct UpdateArgs {
    int rows, cols, rows_p, cols_p;    // as they are, and padded to multiples of 64
    const void *weights, *grad;
    const float *momentum;
    void *weights_out;
    float *momentum_out;
    float beta;
    int nesterov;
    float keep, rate;                  // weights_out = keep weights - rate X
    float eps;
    double *part;                      // [L][kNormBlocks] sums of squares, `parts` of them in use
    int parts;
    _Float16 *Q;                       // planes in the matrix's own order
    _Float16 *T;                       // and transposed
};

constexpr int kNormBlocks = 1024;                  // at most, workgroups of a matrix in the first pass

template <typename E>
__device__ __forceinline__ float momentum_of(const UpdateArgs &p, size_t at)
{
    const float g = to_f32(static_cast<const E *>(p.grad)[at]);
    if (!p.momentum_out) return g;
    const float m = p.momentum_out[at];
    return p.nesterov ? fmaf(p.beta, m, g) : m;
}

// Four entries of a row at a time where they lie at a multiple of their size (FOURS), else one.
template <typename T, bool FOURS>
struct Entries {
    static constexpr int N = FOURS ? 4 : 1;
    typedef T Vec __attribute__((ext_vector_type(4)));
    float v[N];
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (FOURS) {
            const Vec w = *reinterpret_cast<const Vec *>(p);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = to_f32(w[k]);
        } else {
            v[0] = to_f32(*p);
        }
    }
    __device__ __forceinline__ void store(T *p) const
    {
        if constexpr (FOURS) {
            Vec w;
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = from_f32<T>(v[k]);
            *reinterpret_cast<Vec *>(p) = w;
        } else {
            *p = from_f32<T>(v[0]);
        }
    }
};

// The new momentum, and the sum of squares of what is to be orthogonalised (fp64: squares of fp32 do not overflow there).
template <typename E, bool FOURS>
__global__ __launch_bounds__(256) void momentum_kernel(UpdateArgs p)
{
    typedef Entries<E, FOURS> Grad;
    constexpr int N = Grad::N;
    __shared__ double part[256 / kWave];
    const size_t n = (size_t)p.rows * p.cols, base = blockIdx.y * n;
    double sum = 0.0;
#pragma unroll 4
    for (size_t k = ((size_t)blockIdx.x * 256 + threadIdx.x) * N; k < n; k += (size_t)gridDim.x * 256 * N) {
        Grad u;
        u.load(static_cast<const E *>(p.grad) + base + k);
        if (p.momentum) {
            Entries<float, FOURS> m;
            m.load(p.momentum + base + k);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                m.v[e] = fmaf(p.beta, m.v[e], u.v[e]);
                u.v[e] = p.nesterov ? fmaf(p.beta, m.v[e], u.v[e]) : m.v[e];
            }
            m.store(p.momentum_out + base + k);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) sum += (double)u.v[e] * u.v[e];
    }
    for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) p.part[(size_t)blockIdx.y * kNormBlocks + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// 1 / max(norm, eps), times the planes' scale: the parts in fixed order, by a workgroup of 256.  A norm of NaN stays one.
__device__ __forceinline__ double inverse_norm(const UpdateArgs &p, int batch, double *shared)
{
    const double *part = p.part + (size_t)batch * kNormBlocks;
    double sum = 0.0;
    for (int k = threadIdx.x; k < p.parts; k += 256) sum += part[k];
    for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
    if (threadIdx.x % kWave == 0) shared[threadIdx.x / kWave] = sum;
    __syncthreads();
    sum = (shared[0] + shared[1]) + (shared[2] + shared[3]);
    const double norm = sqrt(sum);
    return (double)kPlaneScale / (norm < (double)p.eps ? (double)p.eps : norm);
}

// X = u / max(|u|, eps) as planes, 64 x 64 entries a workgroup, in both orders; padding is zero.
template <typename E>
__global__ __launch_bounds__(256) void planes_kernel(UpdateArgs p)
{
    __shared__ float tile[64][65];
    const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
    const size_t n = (size_t)p.rows * p.cols, base = blockIdx.z * n, padded = (size_t)p.rows_p * p.cols_p * 2 * blockIdx.z;
    __shared__ double shared[256 / kWave];
    const double factor = inverse_norm(p, blockIdx.z, shared);
    for (int k = threadIdx.x; k < 64 * 64; k += 256) {
        const int r = r0 + k / 64, c = c0 + k % 64;
        tile[k / 64][k % 64] = r < p.rows && c < p.cols ? (float)(factor * momentum_of<E>(p, base + (size_t)r * p.cols + c)) : 0.0f;
    }
    __syncthreads();
    auto put = [&](_Float16 *Q, size_t row, int ld, int c, const float *v) {
        half8 h, l;
        for (int e = 0; e < 8; ++e) {
            h[e] = (_Float16)v[e];
            l[e] = (_Float16)(v[e] - (float)h[e]);
        }
        _Float16 *to = Q + padded + row * ld * 2 + plane_at(c);
        *reinterpret_cast<half8 *>(to) = h;
        *reinterpret_cast<half8 *>(to + 32) = l;
    };
    for (int k = threadIdx.x; k < 64 * 8; k += 256) {
        const int r = k / 8, c = k % 8 * 8;
        float v[8], w[8];
        for (int e = 0; e < 8; ++e) {
            v[e] = tile[r][c + e];
            w[e] = tile[c + e][r];
        }
        put(p.Q, (size_t)r0 + r, p.cols_p, c0 + c, v);
        put(p.T, (size_t)c0 + r, p.rows_p, r0 + c, w);
    }
}

// The update by X as it started: no step at all.  (Otherwise the last product writes the matrix.)
template <typename E, bool FOURS>
__global__ __launch_bounds__(256) void finish_kernel(UpdateArgs p)
{
    constexpr int N = FOURS ? 4 : 1;
    const size_t n = (size_t)p.rows * p.cols, base = blockIdx.y * n, padded = (size_t)p.rows_p * p.cols_p * 2 * blockIdx.y;
    for (size_t k = ((size_t)blockIdx.x * 256 + threadIdx.x) * N; k < n; k += (size_t)gridDim.x * 256 * N) {
        const int r = (int)(k / p.cols), c = (int)(k % p.cols);        // FOURS: rows are multiples of four
        const size_t at = padded + (size_t)r * p.cols_p * 2 + plane_at(c);
        Entries<_Float16, FOURS> h, l;
        h.load(p.Q + at);
        l.load(p.Q + at + 32);
        Entries<E, FOURS> w;
        if (p.weights) w.load(static_cast<const E *>(p.weights) + base + k);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float x = (h.v[e] + l.v[e]) * (1.0f / kPlaneScale);
            w.v[e] = p.weights ? p.keep * w.v[e] - p.rate * x : x;
        }
        w.store(static_cast<E *>(p.weights_out) + base + k);
    }
}

bool sizes_ok(int L, int rows, int cols) { return L >= 0 && L <= 65535 && rows >= 1 && cols >= 1 && rows <= 32768 && cols <= 32768; }

size_t up(size_t n) { return (n + 255) / 256 * 256; }

// ---- which tiles a product takes
struct Plan { int shape, splits; };                // shape: 0 of 256 x 256, 1 of 128 x 128, 2 of 64 x 64 results, 3 as 1 by two groups of waves

constexpr int kSide[4] = {256, 128, 64, 128};

int tiles_of(int shape, int Mp, int Np, bool symmetric)
{
    const int tm = (Mp + kSide[shape] - 1) / kSide[shape], tn = (Np + kSide[shape] - 1) / kSide[shape];
    return symmetric ? tm * (tm + 1) / 2 : tm * tn;
}

Plan plan_of(int L, int Mp, int Np, bool symmetric, int stages)
{
    // The largest tile of which half the compute units get one.  A G or P that still leaves compute units without one and is long
    // enough to pay for a second pass over its sums (2048 x 8192, G: 134 us, 179 in one part; 4096 x 4096, G and P: 236, 248) goes in parts.
    Plan best{2, 1};
    for (int shape = 0; shape < 3; ++shape)
        if ((int64_t)tiles_of(shape, Mp, Np, symmetric) * L >= 128) { best.shape = shape; break; }
    const int64_t tiles = (int64_t)tiles_of(best.shape, Mp, Np, symmetric) * L;
    if (symmetric && stages >= 128 && tiles < 256) best.splits = (int)std::max<int64_t>(1, std::min<int64_t>(512 / tiles, stages / 16));
    // One 128 x 128 tile on a compute unit: two groups of waves, each with half of the sum, keep it busier than one (2048 x 2048 fp32:
    // 3 us less a G or P, 6 an X; with more tiles two workgroups do that).
    if (best.shape == 1 && best.splits == 1 && tiles <= 256) best.shape = 3;
    return best;
}

struct Layout {
    int rows_p, cols_p, s, l, s_p, l_p;
    size_t x[2], t[2], g, p, part, partial, bytes;
};

Layout layout_of(int L, int rows, int cols)
{
    Layout y{};
    if (small_fits(rows, cols)) { y.bytes = 256; return y; }   // shared memory alone; a size of zero would be a special case for callers
    auto pad = [](int v) { return (v + 63) / 64 * 64; };
    y.rows_p = pad(rows); y.cols_p = pad(cols);
    y.s = rows < cols ? rows : cols; y.l = rows < cols ? cols : rows;
    y.s_p = pad(y.s); y.l_p = pad(y.l);
    const size_t n = (size_t)L * y.rows_p * y.cols_p * 2 * sizeof(_Float16), square = (size_t)L * y.s_p * y.s_p * 2 * sizeof(_Float16);
    size_t at = 0, partial = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += up(bytes); return here; };
    for (int k = 0; k < 2; ++k) {
        y.x[k] = take(n);
        y.t[k] = take(n);
    }
    y.g = take(square);
    y.p = take(square);
    y.part = take((size_t)L * kNormBlocks * sizeof(double));
    const int stages_g = y.l_p / 32, stages_p = y.s_p / 32;
    for (int stages : {stages_g, stages_p}) {
        const Plan plan = plan_of(L, y.s_p, y.s_p, true, stages);
        if (plan.splits > 1)
            partial = std::max(partial, (size_t)L * tiles_of(plan.shape, y.s_p, y.s_p, true) * plan.splits * kSide[plan.shape] * kSide[plan.shape] * sizeof(float));
    }
    y.partial = take(partial);
    y.bytes = at;
    return y;
}

template <class S, typename E>
int launch_product(Product p, int L, hipStream_t stream)
{
    static_assert(S::kLds <= 160 * 1024, "");
    p.tiles_m = (p.Mp + S::TM - 1) / S::TM;
    p.tiles_n = (p.Np + S::TN - 1) / S::TN;
    p.tiles = p.symmetric ? p.tiles_m * (p.tiles_m + 1) / 2 : p.tiles_m * p.tiles_n;
    if constexpr (S::kLds > 64 * 1024) {
        for (const void *k : {reinterpret_cast<const void *>(product_kernel<S, E>), reinterpret_cast<const void *>(join_kernel<S, E>)}) {
            const hipError_t err = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds);
            if (err != hipSuccess) return report_device_error(err, "hipFuncSetAttribute");
        }
    }
    hipLaunchKernelGGL((product_kernel<S, E>), dim3((unsigned)(p.tiles * p.splits), (unsigned)L), dim3(S::kThreads), S::kLds, stream, p);
    if (p.splits > 1) hipLaunchKernelGGL((join_kernel<S, E>), dim3((unsigned)p.tiles, (unsigned)L, S::NT * S::MT / kJoinBlocks<S>), dim3(S::kTileThreads), S::kWaves * S::staging(kJoinBlocks<S>), stream, p);
    return MARL_OK;
}

template <typename E>
int product(Product p, int L, hipStream_t stream)
{
    const Plan plan = plan_of(L, p.Mp, p.Np, p.symmetric, p.stages);
    p.splits = plan.splits;
    switch (plan.shape) {
    case 0: return launch_product<TileShape<2, 4, 4, 2, 2>, E>(p, L, stream);
    case 1: return launch_product<TileShape<2, 2, 2, 2, 2>, E>(p, L, stream);
    case 2: return launch_product<TileShape<2, 2, 1, 1, 4>, E>(p, L, stream);
    default: return launch_product<TileShape<2, 2, 2, 2, 2, 2>, E>(p, L, stream);
    }
}

template <typename E>
int iterate(const Layout &y, int L, UpdateArgs p, char *workspace, int steps, const float *coef, hipStream_t stream)
{
    auto at = [&](size_t offset) { return reinterpret_cast<_Float16 *>(workspace + offset); };
    const bool tall = p.rows > p.cols;
    _Float16 *X[2], *T[2];                           // X [s][l] and its transpose
    for (int k = 0; k < 2; ++k) {
        X[k] = at(y.x[k]);
        T[k] = at(y.t[k]);
    }
    p.rows_p = y.rows_p; p.cols_p = y.cols_p;
    p.part = reinterpret_cast<double *>(workspace + y.part);
    p.Q = tall ? T[0] : X[0];
    p.T = tall ? X[0] : T[0];
    const size_t n = (size_t)p.rows * p.cols;
    const bool fours = p.cols % 4 == 0 && aligned_to(p.grad, 4 * sizeof(E)) && aligned_to(p.weights, 4 * sizeof(E)) &&
                       aligned_to(p.weights_out, 4 * sizeof(E)) && aligned_to(p.momentum, 16) && aligned_to(p.momentum_out, 16);
    // four entries a thread and turn, four turns; the passes over the entries are bound by their bytes
    const unsigned blocks = (unsigned)std::min<size_t>(kNormBlocks, (n + 256 * 16 - 1) / (256 * 16));
    p.parts = (int)blocks;
    if (fours) hipLaunchKernelGGL((momentum_kernel<E, true>), dim3(blocks, (unsigned)L), dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((momentum_kernel<E, false>), dim3(blocks, (unsigned)L), dim3(256), 0, stream, p);
    hipLaunchKernelGGL((planes_kernel<E>), dim3((unsigned)(y.cols_p / 64), (unsigned)(y.rows_p / 64), (unsigned)L), dim3(256), 0, stream, p);
    const int64_t square = (int64_t)y.s_p * y.s_p * 2, whole = (int64_t)y.s_p * y.l_p * 2;
    int now = 0;
    for (int k = 0; k < steps; ++k) {
        Product g{};
        g.A = g.B = X[now]; g.a_batch = g.b_batch = whole; g.lda = g.ldb = (int64_t)y.l_p * 2;
        g.Mp = g.Np = y.s_p; g.stages = y.l_p / 32;
        g.alpha = 1.0f / kPlaneScale;
        g.Dt = g.D = at(y.g); g.ldt = g.ldd = (int64_t)y.s_p * 2; g.t_batch = g.d_batch = square;
        g.symmetric = 1;
        g.partial = reinterpret_cast<float *>(workspace + y.partial);
        int rc = product<E>(g, L, stream);
        if (rc) return rc;
        Product q = g;
        q.A = q.B = at(y.g); q.a_batch = q.b_batch = square; q.lda = q.ldb = (int64_t)y.s_p * 2;
        q.stages = y.s_p / 32;
        q.alpha = coef[2] / kPlaneScale; q.beta = coef[1];
        q.C = at(y.g);
        q.Dt = q.D = at(y.p);
        rc = product<E>(q, L, stream);
        if (rc) return rc;
        Product x{};                                   // D [l][s] = X^T P, so D's transpose is the new X
        x.A = T[now]; x.a_batch = whole; x.lda = (int64_t)y.s_p * 2;
        x.B = at(y.p); x.b_batch = square; x.ldb = (int64_t)y.s_p * 2;
        x.Mp = y.l_p; x.Np = y.s_p; x.stages = y.s_p / 32;
        x.alpha = 1.0f / kPlaneScale; x.beta = coef[0];
        x.C = X[now];
        x.Dt = X[now ^ 1]; x.ldt = (int64_t)y.l_p * 2; x.t_batch = whole;
        x.D = T[now ^ 1]; x.ldd = (int64_t)y.s_p * 2; x.d_batch = whole;
        if (k + 1 == steps) {
            x.out = p.weights_out; x.weights = p.weights;
            x.rows = p.rows; x.cols = p.cols; x.tall = tall; x.keep = p.keep; x.rate = p.rate;
        }
        rc = product<E>(x, L, stream);
        if (rc) return rc;
        now ^= 1;
    }
    if (steps == 0) {
        const dim3 each((unsigned)std::min<size_t>((n + 1023) / 1024, 4096), (unsigned)L);
        if (fours) hipLaunchKernelGGL((finish_kernel<E, true>), each, dim3(256), 0, stream, p);
        else hipLaunchKernelGGL((finish_kernel<E, false>), each, dim3(256), 0, stream, p);
    }
    return launched("orthogonalised update");
}

template <typename E>
int iterate_small(int L, const UpdateArgs &p, int steps, const float *coef, hipStream_t stream)
{
    const int bytes = small_shape(p.rows, p.cols).bytes;
    const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(small_kernel<E>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (err != hipSuccess) return report_device_error(err, "hipFuncSetAttribute");
    const SmallArgs a{p.rows, p.cols, steps, p.nesterov, p.weights, p.grad, p.momentum, p.weights_out, p.momentum_out,
                      p.beta, p.keep, p.rate, p.eps, coef[0], coef[1], coef[2]};
    hipLaunchKernelGGL(small_kernel<E>, dim3((unsigned)L), dim3(kSmallThreads), bytes, stream, a);
    return launched("orthogonalised update");
}

int newton_schulz(int dtype, int L, UpdateArgs p, char *workspace, int steps, const float *coef, float eps, hipStream_t stream)
{
    p.eps = eps;
    if (small_fits(p.rows, p.cols)) return with_dtype(dtype, [&](auto e) { return iterate_small<decltype(e)>(L, p, steps, coef, stream); });
    const Layout y = layout_of(L, p.rows, p.cols);
    return with_dtype(dtype, [&](auto e) { return iterate<decltype(e)>(y, L, p, workspace, steps, coef, stream); });
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
