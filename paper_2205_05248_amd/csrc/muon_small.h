// The whole Newton-Schulz iteration of a small matrix in one workgroup: X, its transpose, G and P stay in shared memory.
// A product of such a matrix takes a microsecond and a launch costs more: three products a step and the two passes around them
// were 18 launches and 83 us for two matrices of 192 x 64.  Tiles of 16 x 16, one per wave and turn, sixteen waves: the chain of
// dependent matrix instructions, which is what bounds it, is as short as it gets.  Planes as in muon_product.h.
#pragma once
#include "muon_product.h"

namespace marl {

// What a thread and a wave hold at most: entries of the matrix, tiles of X.  Both planes of X and of its transpose in 160 KB leave
// no more than 20480 entries.
constexpr int kSmallThreads = 1024, kSmallEntries = 20, kSmallTurns = 5;

// Rows of planes in shared memory: 16 bytes more than a multiple of 128, so that sixteen rows meet all banks.
__host__ __device__ __forceinline__ int small_row(int k) { return 2 * k + 8; }

struct SmallShape {
    int s, l;                          // short and long side, padded to multiples of 32
    int x, t, g, p, bytes;             // offsets in fp16 values, and bytes of all
};

__host__ __device__ inline SmallShape small_shape(int rows, int cols)
{
    SmallShape y{};
    const int s = rows < cols ? rows : cols, l = rows < cols ? cols : rows;
    y.s = (s + 31) / 32 * 32;
    y.l = (l + 31) / 32 * 32;
    y.x = 0;
    y.t = y.x + y.s * small_row(y.l);
    y.g = y.t + y.l * small_row(y.s);
    y.p = y.g + y.s * small_row(y.s);
    y.bytes = (y.p + y.s * small_row(y.s)) * 2;
    return y;
}

inline bool small_fits(int rows, int cols)
{
    if ((int64_t)rows * cols > kSmallEntries * kSmallThreads) return false;
    const SmallShape y = small_shape(rows, cols);
    const int waves = kSmallThreads / kWave, ts = y.s / 16;
    return y.bytes <= 159 * 1024 && ts <= waves && y.l / 16 <= kSmallTurns * (waves / ts);
}

struct SmallArgs {
    int rows, cols, steps, nesterov;
    const void *weights, *grad;
    const float *momentum;
    void *weights_out;
    float *momentum_out;
    float beta, keep, rate, eps, c0, c1, c2;
};

template <typename E>
__global__ __launch_bounds__(kSmallThreads) void small_kernel(SmallArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ double part[kSmallThreads / kWave];
    _Float16 *planes = reinterpret_cast<_Float16 *>(lds);
    const SmallShape y = small_shape(a.rows, a.cols);
    const bool tall = a.rows > a.cols;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), n = a.rows * a.cols;
    const size_t base = (size_t)blockIdx.x * n;
    _Float16 *X = planes + y.x, *T = planes + y.t, *G = planes + y.g, *P = planes + y.p;
    const int ldx = small_row(y.l), lds_s = small_row(y.s);

    float u[kSmallEntries];                                // momentum, or the gradient alone
    double sum = 0.0;
#pragma unroll
    for (int q = 0; q < kSmallEntries; ++q) {
        const int k = threadIdx.x + q * kSmallThreads;
        u[q] = k < n ? to_f32(static_cast<const E *>(a.grad)[base + k]) : 0.0f;
    }
    if (a.momentum) {
        float m[kSmallEntries];
#pragma unroll
        for (int q = 0; q < kSmallEntries; ++q) {
            const int k = threadIdx.x + q * kSmallThreads;
            m[q] = k < n ? a.momentum[base + k] : 0.0f;
        }
#pragma unroll
        for (int q = 0; q < kSmallEntries; ++q) {
            const int k = threadIdx.x + q * kSmallThreads;
            m[q] = fmaf(a.beta, m[q], u[q]);
            if (k < n) a.momentum_out[base + k] = m[q];
            u[q] = a.nesterov ? fmaf(a.beta, m[q], u[q]) : m[q];
        }
    }
#pragma unroll
    for (int q = 0; q < kSmallEntries; ++q) sum += (double)u[q] * u[q];
    for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
    if (lane == 0) part[wave] = sum;
    for (int k = threadIdx.x; k < y.g / 8; k += kSmallThreads) reinterpret_cast<half8 *>(planes)[k] = half8{};     // padding of X and T
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < kSmallThreads / kWave; ++w) sum += part[w];
    const double norm = sqrt(sum), factor = (double)kPlaneScale / (norm < (double)a.eps ? (double)a.eps : norm);         // (a norm of NaN stays one)
    auto put = [&](_Float16 *to, float v) {
        const _Float16 h = (_Float16)v;
        to[0] = h;
        to[32] = (_Float16)(v - (float)h);
    };
    // n < 2^15: the reciprocal, rounded up, gives the row without a division
    const unsigned per_row = (unsigned)(0xffffffffu / (unsigned)a.cols) + 1;
    auto row_of = [&](int k) { return a.cols == 1 ? k : (int)__umulhi((unsigned)k, per_row); };
#pragma unroll
    for (int q = 0; q < kSmallEntries; ++q) {
        const int k = threadIdx.x + q * kSmallThreads, r = row_of(k), c = k - r * a.cols;
        if (k >= n) break;
        const float v = (float)(factor * u[q]);
        const int i = tall ? c : r, j = tall ? r : c;      // X[i][j]
        put(X + i * ldx + plane_at(j), v);
        put(T + j * lds_s + plane_at(i), v);
    }
    __syncthreads();

    // 16 x 16 results of A B^T over K: rows 4 (lane / 16) + e of A, row lane % 16 of B.  Of N tiles below one another, `down` rows
    // of A apart, those there are: what bounds it is shared memory, and they share the reads of B.
    auto tiles = [&](auto count, int there, const _Float16 *A, int lda, int m0, int down, const _Float16 *B, int ldb, int n0, int K, floatx4 *out) {
        constexpr int N = decltype(count)::value;
        constexpr int kSpan = 64;                           // terms of a sum by themselves, as in muon_product.h (only G's are long)
        floatx4 cross[N], total = {0, 0, 0, 0};
#pragma unroll
        for (int q = 0; q < N; ++q) out[q] = cross[q] = floatx4{0, 0, 0, 0};
        const _Float16 *pa = A + (m0 + (lane & 15)) * lda + 8 * (lane >> 4), *pb = B + (n0 + (lane & 15)) * ldb + 8 * (lane >> 4);
        for (int k = 0; k < K; k += 32) {
            if constexpr (N == 1)
                if (k > 0 && k % kSpan == 0) {
                    total += out[0];
                    out[0] = floatx4{0, 0, 0, 0};
                }
            const half8 bh = *reinterpret_cast<const half8 *>(pb + 2 * k), bl = *reinterpret_cast<const half8 *>(pb + 2 * k + 32);
#pragma unroll
            for (int q = 0; q < N; ++q)
                if (q < there) {
                    const _Float16 *at = pa + q * down * lda + 2 * k;
                    const half8 ah = *reinterpret_cast<const half8 *>(at), al = *reinterpret_cast<const half8 *>(at + 32);
                    out[q] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, bh, out[q], 0, 0, 0);
                    cross[q] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, bl, cross[q], 0, 0, 0);
                    cross[q] = __builtin_amdgcn_mfma_f32_16x16x32_f16(al, bh, cross[q], 0, 0, 0);
                }
        }
#pragma unroll
        for (int q = 0; q < N; ++q) out[q] += total + cross[q];
    };
    auto put_along = [&](_Float16 *to, const floatx4 &v) {  // four entries along a row
        half4 h, l;
        for (int e = 0; e < 4; ++e) {
            h[e] = (_Float16)v[e];
            l[e] = (_Float16)(v[e] - (float)h[e]);
        }
        *reinterpret_cast<half4 *>(to) = h;
        *reinterpret_cast<half4 *>(to + 32) = l;
    };
    const int ts = y.s / 16, waves = kSmallThreads / kWave;
    const int m4 = 4 * (lane >> 4), nn = lane & 15;
    // a symmetric matrix: tiles on and below the diagonal, and their mirror images
    auto square = [&](const _Float16 *A, int lda, int K, _Float16 *D, float alpha, float beta) {
        for (int k = wave; k < ts * (ts + 1) / 2; k += waves) {
            int i = 0;
            while ((i + 1) * (i + 2) / 2 <= k) ++i;
            const int m0 = i * 16, n0 = (k - i * (i + 1) / 2) * 16;
            floatx4 v;
            tiles(std::integral_constant<int, 1>{}, 1, A, lda, m0, 0, A, lda, n0, K, &v);
            const int at = (n0 + nn) * lds_s + plane_at(m0 + m4);
            v *= alpha;
            if (beta != 0.0f) {
                const half4 h = *reinterpret_cast<const half4 *>(G + at), l = *reinterpret_cast<const half4 *>(G + at + 32);
                for (int e = 0; e < 4; ++e) v[e] = fmaf(beta, (float)h[e] + (float)l[e], v[e]);
            }
            put_along(D + at, v);
            if (m0 != n0)
                for (int e = 0; e < 4; ++e) put(D + (m0 + m4 + e) * lds_s + plane_at(n0 + nn), v[e]);
        }
        __syncthreads();
    };
    // D [l][s] = T P: a wave has one column of tiles and every `side`-th row of them
    const int side = waves / ts, n0 = wave % ts * 16, i0 = wave / ts, rows_of_tiles = y.l / 16;
    const int there = i0 < side && i0 < rows_of_tiles ? (rows_of_tiles - i0 + side - 1) / side : 0;
    for (int step = 0; step < a.steps; ++step) {
        square(X, ldx, y.l, G, 1.0f / kPlaneScale, 0.0f);
        square(G, lds_s, y.s, P, a.c2 / kPlaneScale, a.c1);
        floatx4 held[kSmallTurns];                          // all of D is formed before any of X is overwritten
        if (there) tiles(std::integral_constant<int, kSmallTurns>{}, there, T, lds_s, i0 * 16, side * 16, P, lds_s, n0, y.s, held);
#pragma unroll
        for (int q = 0; q < kSmallTurns; ++q)
            if (q < there) {
                const int at = (n0 + nn) * ldx + plane_at((i0 + q * side) * 16 + m4);
                const half4 h = *reinterpret_cast<const half4 *>(X + at), l = *reinterpret_cast<const half4 *>(X + at + 32);
                for (int e = 0; e < 4; ++e) held[q][e] = fmaf(a.c0, (float)h[e] + (float)l[e], held[q][e] * (1.0f / kPlaneScale));
            }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kSmallTurns; ++q)
            if (q < there) {
                const int m0 = (i0 + q * side) * 16;
                put_along(X + (n0 + nn) * ldx + plane_at(m0 + m4), held[q]);
                for (int e = 0; e < 4; ++e) put(T + (m0 + m4 + e) * lds_s + plane_at(n0 + nn), held[q][e]);
            }
        __syncthreads();
    }
#pragma unroll
    for (int q = 0; q < kSmallEntries; ++q) {
        const int k = threadIdx.x + q * kSmallThreads;
        u[q] = a.weights && k < n ? to_f32(static_cast<const E *>(a.weights)[base + k]) : 0.0f;
    }
#pragma unroll
    for (int q = 0; q < kSmallEntries; ++q) {
        const int k = threadIdx.x + q * kSmallThreads, r = row_of(k), c = k - r * a.cols;
        if (k >= n) break;
        const _Float16 *at = tall ? T + r * lds_s + plane_at(c) : X + r * ldx + plane_at(c);
        const float x = ((float)at[0] + (float)at[32]) * (1.0f / kPlaneScale);
        static_cast<E *>(a.weights_out)[base + k] = from_f32<E>(a.weights ? a.keep * u[q] - a.rate * x : x);
    }
}

}  // namespace marl
