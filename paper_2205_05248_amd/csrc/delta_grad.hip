// Gated delta rule, backward: the way back through the chunks, then the gradients of every chunk side by side.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "delta.h"

namespace marl {
namespace {

// The chunks of one head from the last to the first, for kCols value columns: D, Y and the gradient of v.  Wave w has rows 16 w
// on of the chunk, and rows w DK / 4 on of the adjoint, which stays in its accumulators.
template <typename E, int DK>
__global__ __launch_bounds__(kDeltaThreads) void back_kernel(DeltaArgs p)
{
    constexpr int LD = DK + 1, LS = DK + 1, LU = kSteps + 1;
    constexpr int kTiles = (DK + 63) / 64;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    float *K = lds, *Q = K + kSteps * LD, *S = Q + kSteps * LD, *O = S + kCols * LS, *R = O + kCols * LU, *V = R + kCols * LU;
    __shared__ ChunkGates gates;
    __shared__ int not_finite[2];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, at = lane % 16, group = lane / 16;
    const int blocks = (p.Dv + kCols - 1) / kCols;
    const int64_t head = blockIdx.x / blocks;
    const int first = (int)(blockIdx.x % blocks) * kCols, col = first + at;
    const int h = (int)(head % p.Hv), hk = h / (p.Hv / p.Hk);
    const int64_t b = head / p.Hv;
    const bool in = col < p.Dv;
    Acc adj[kTiles];
    auto key_row = [&](int tile, int r) { return (wave * kTiles + tile) * 16 + group * 4 + r; };
#pragma unroll
    for (int tile = 0; tile < kTiles; ++tile)
        for (int r = 0; r < 4; ++r) {
            const int d = key_row(tile, r);
            adj[tile][r] = p.grad_s_last && in && d < p.Dk ? p.grad_s_last[(head * p.Dk + d) * p.Dv + col] : 0.0f;
        }
    for (int chunk = p.chunks - 1; chunk >= 0; --chunk) {
        const int64_t record = head * p.chunks + chunk;
        __syncthreads();
        {
            const int *from = reinterpret_cast<const int *>(p.gates + record);
            int *to = reinterpret_cast<int *>(&gates);
            for (int e = threadIdx.x; e < (int)(sizeof(ChunkGates) / 4); e += kDeltaThreads) to[e] = from[e];
        }
        if (threadIdx.x < 2) not_finite[threadIdx.x] = 0;
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile)
            for (int r = 0; r < 4; ++r) {
                const int d = key_row(tile, r);
                if (d < DK) S[at * LS + d] = adj[tile][r];
                if (in && d < p.Dk) p.D[(record * p.Dk + d) * p.Dv + col] = adj[tile][r];
            }
        __syncthreads();
        const unsigned long long starts = gates.starts, alive = gates.live;
        for (int e = threadIdx.x; e < kSteps * DK; e += kDeltaThreads) {
            const int i = e / DK, d = e % DK;
            const bool is = bit_of(alive, i) && d < p.Dk;
            K[i * LD + d] = is ? to_f32(row_at<E>(p.k, p.ld_k, b, p.T, chunk * kSteps + i, hk, p.Dk)[d]) : 0.0f;
            Q[i * LD + d] = is ? to_f32(row_at<E>(p.q, p.ld_q, b, p.T, chunk * kSteps + i, hk, p.Dk)[d]) : 0.0f;
        }
        Acc go, scaled, y;
        for (int r = 0; r < 4; ++r) {
            const int i = wave * 16 + group * 4 + r;
            go[r] = bit_of(alive, i) && in ? to_f32(row_at<E>(p.grad_o, p.ld_go, b, p.T, chunk * kSteps + i, h, p.Dv)[col]) : 0.0f;
            O[at * LU + i] = go[r];
        }
        if (!all_finite(go)) not_finite[0] = 1;
        __syncthreads();
        // dU = P' dO + t K D
        Acc kd = {};
        kd = product(DK, kd, [&](int row, int k) { return K[(wave * 16 + row) * LD + k]; }, [&](int k, int c) { return S[c * LS + k]; });
        for (int r = 0; r < 4; ++r) {
            const int i = wave * 16 + group * 4 + r;
            const float t = gates.t[i];
            y[r] = t == 0.0f || !bit_of(alive, i) ? 0.0f : t * kd[r];
        }
        const float *P = p.P + record * kSteps * kSteps + wave * 16, *N = p.N + record * kSteps * kSteps + wave * 16;
        auto of_p = [&](int row, int k) { return P[k * kSteps + row]; };
        auto of_o = [&](int k, int c) { return O[c * LU + k]; };
        if (gates.bad || not_finite[0])
            y = careful_product(kSteps, y, of_p, of_o, [&](int row, int k) {
                const int i = wave * 16 + row;
                return k >= i && bit_of(alive, i) && bit_of(alive, k) && joined(starts, k, i);
            });
        else y = product(kSteps - wave * 16, y, [&](int row, int k) { return of_p(row, wave * 16 + k); }, [&](int k, int c) { return of_o(wave * 16 + k, c); });
        // Y = dU - N' (beta dU)
        for (int r = 0; r < 4; ++r) {
            const int i = wave * 16 + group * 4 + r;
            scaled[r] = bit_of(alive, i) ? gates.beta[i] * y[r] : 0.0f;
            R[at * LU + i] = scaled[r];
        }
        if (!all_finite(scaled)) not_finite[1] = 1;
        __syncthreads();
        auto of_n = [&](int row, int k) { return -N[k * kSteps + row]; };
        auto of_r = [&](int k, int c) { return R[c * LU + k]; };
        if (gates.bad || not_finite[1])
            y = careful_product(kSteps, y, of_n, of_r, [&](int row, int k) {
                const int i = wave * 16 + row;
                return k > i && bit_of(alive, i) && bit_of(alive, k) && joined(starts, k, i);
            });
        else y = product(kSteps - wave * 16, y, [&](int row, int k) { return of_n(row, wave * 16 + k); }, [&](int k, int c) { return of_r(wave * 16 + k, c); });
        for (int r = 0; r < 4; ++r) {
            const int i = wave * 16 + group * 4 + r, t = chunk * kSteps + i;
            const float v = bit_of(alive, i) ? gates.beta[i] * y[r] : 0.0f;
            const float f = gates.f[i];
            V[at * LU + i] = f == 0.0f ? 0.0f : -f * v;
            O[at * LU + i] = f == 0.0f ? 0.0f : p.scale * f * go[r];       // the wave's own rows, which others read before the barrier above
            if (in) p.Y[(record * kSteps + i) * p.Dv + col] = bit_of(alive, i) ? y[r] : 0.0f;
            if (t < p.T && in) const_cast<E *>(row_at<E>(p.grad_v, p.ld_gv, b, p.T, t, h, p.Dv))[col] = from_f32<E>(v);
        }
        __syncthreads();
        // D <- f_63 D + (scale f Q)' dO - (f K)' dV
        const float whole = gates.f[kSteps - 1];
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile) {
            for (int r = 0; r < 4; ++r) adj[tile][r] = whole == 0.0f ? 0.0f : whole * adj[tile][r];
            const int d0 = (wave * kTiles + tile) * 16;
            if (d0 < DK) {
                adj[tile] = product(kSteps, adj[tile], [&](int row, int k) { return gates.f[k] == 0.0f ? 0.0f : Q[k * LD + d0 + row]; },
                                    [&](int k, int c) { return O[c * LU + k]; });
                adj[tile] = product(kSteps, adj[tile], [&](int row, int k) { return gates.f[k] == 0.0f ? 0.0f : K[k * LD + d0 + row]; },
                                    [&](int k, int c) { return V[c * LU + k]; });
            }
        }
    }
    if (p.grad_s_first)
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile)
            for (int r = 0; r < 4; ++r) {
                const int d = key_row(tile, r);
                if (in && d < p.Dk) p.grad_s_first[(head * p.Dk + d) * p.Dv + col] = adj[tile][r];
            }
}

// Sum over the 16 lanes that hold a row.
__device__ __forceinline__ float row_sum(float v)
{
    for (int d = 1; d < 16; d *= 2) v += __shfl_xor(v, d);
    return v;
}

// Gradients of q, k, beta and the log decay of a chunk, the value heads of a key head one after the other.  Wave w has rows 16 w
// on.  With dP = scale dO U', dA = -(dV) U' and their products with E, dN and dM:
//   dq = dN K + scale f dO S'      dk = [dM K - f dV S'] + [dN' Q + dM' K + t U D']
//   dG_i = q_i.dq_i + k_i.[first] - k_i.[second], to which the last step adds sum_j k_j.(t U D')_j + f_63 <D, S>;
// the log decay's gradient is the sum of dG from its step to the end of its sequence.
template <typename E, int DK>
__global__ __launch_bounds__(kDeltaThreads) void chunk_grad_kernel(DeltaArgs p)
{
    constexpr int LD = DK + 1, LN = kSteps + 1, kTiles = DK / 16;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    float *K = lds, *Q = K + kSteps * LD, *dN = Q + kSteps * LD, *dM = dN + kSteps * LN;
    __shared__ ChunkGates gates;
    __shared__ int not_finite;
    __shared__ float dG[kSteps], extra[kDeltaThreads / kWave], dbeta[kSteps];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, at = lane % 16, group = lane / 16;
    const int chunk = (int)(blockIdx.x % p.chunks), hk = (int)(blockIdx.x / p.chunks % p.Hk);
    const int64_t b = blockIdx.x / p.chunks / p.Hk;
    const int shared = p.Hv / p.Hk;
    Acc sum_q[kTiles] = {}, sum_k[kTiles] = {};
    for (int member = 0; member < shared; ++member) {
        const int h = hk * shared + member;
        const int64_t record = (b * p.Hv + h) * p.chunks + chunk;
        __syncthreads();
        {
            const int *from = reinterpret_cast<const int *>(p.gates + record);
            int *to = reinterpret_cast<int *>(&gates);
            for (int e = threadIdx.x; e < (int)(sizeof(ChunkGates) / 4); e += kDeltaThreads) to[e] = from[e];
        }
        if (threadIdx.x == 0) not_finite = 0;
        __syncthreads();
        const unsigned long long starts = gates.starts, alive = gates.live;
        if (member == 0)
            for (int e = threadIdx.x; e < kSteps * DK; e += kDeltaThreads) {
                const int i = e / DK, d = e % DK;
                const bool is = bit_of(alive, i) && d < p.Dk;
                K[i * LD + d] = is ? to_f32(row_at<E>(p.k, p.ld_k, b, p.T, chunk * kSteps + i, hk, p.Dk)[d]) : 0.0f;
                Q[i * LD + d] = is ? to_f32(row_at<E>(p.q, p.ld_q, b, p.T, chunk * kSteps + i, hk, p.Dk)[d]) : 0.0f;
            }
        const float *M = p.M + record * kSteps * p.Dv, *Y = p.Y + record * kSteps * p.Dv;
        const float *S = p.S + record * p.Dk * p.Dv, *D = p.D + record * p.Dk * p.Dv;
        auto grad_o = [&](int i, int c) {
            return bit_of(alive, i) && c < p.Dv ? to_f32(row_at<E>(p.grad_o, p.ld_go, b, p.T, chunk * kSteps + i, h, p.Dv)[c]) : 0.0f;
        };
        auto grad_v = [&](int i, int c) { return bit_of(alive, i) && c < p.Dv ? gates.beta[i] * Y[i * p.Dv + c] : 0.0f; };
        auto u = [&](int i, int c) { return bit_of(alive, i) && c < p.Dv ? gates.beta[i] * M[i * p.Dv + c] : 0.0f; };
        auto mine = [&](int row) { return wave * 16 + row; };
        bool fine = true;
        for (int tile = 0; tile < 4; ++tile) {
            Acc n = {}, m = {};
            if (tile <= wave) {
                auto of_u = [&](int k, int c) { return u(tile * 16 + c, k); };
                n = product((p.Dv + 3) / 4 * 4, n, [&](int row, int k) { return grad_o(mine(row), k); }, of_u);
                m = product((p.Dv + 3) / 4 * 4, m, [&](int row, int k) { return -grad_v(mine(row), k); }, of_u);
            }
            const int j = tile * 16 + at;
            for (int r = 0; r < 4; ++r) {
                const int i = mine(group * 4 + r);
                const bool on = j <= i && bit_of(alive, i) && bit_of(alive, j) && joined(starts, i, j);
                const float e = on ? decay_of(gates.G[i] - gates.G[j]) : 0.0f;
                const float a = on ? p.scale * e * n[r] : 0.0f, c = on && j < i ? e * m[r] : 0.0f;
                dN[i * LN + j] = a;
                dM[i * LN + j] = c;
                fine = fine && (a + c) * 0.0f == 0.0f;
            }
        }
        for (int e = threadIdx.x; member == 0 && e < kSteps * DK; e += kDeltaThreads) fine = fine && (K[e / DK * LD + e % DK] + Q[e / DK * LD + e % DK]) * 0.0f == 0.0f;
        if (!fine) not_finite = 1;
        // dbeta = M.Y, four lanes a row
        {
            const int i = threadIdx.x / 4;
            float v = 0.0f;
            if (bit_of(alive, i))
                for (int c = threadIdx.x % 4; c < p.Dv; c += 4) v = fmaf(M[i * p.Dv + c], Y[i * p.Dv + c], v);
            v += __shfl_xor(v, 1);
            v += __shfl_xor(v, 2);
            if (threadIdx.x % 4 == 0) dbeta[i] = v;
        }
        __syncthreads();
        const bool bad = gates.bad || not_finite;
        Acc dq[kTiles], plus[kTiles], minus[kTiles];
        float at_end = 0.0f, dot[4] = {};
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile) {
            const int d = tile * 16 + at, n = (p.Dv + 3) / 4 * 4;
            auto of_s = [&](int k, int c) { return tile * 16 + c < p.Dk && k < p.Dv ? S[(tile * 16 + c) * p.Dv + k] : 0.0f; };
            auto of_d = [&](int k, int c) { return tile * 16 + c < p.Dk && k < p.Dv ? D[(tile * 16 + c) * p.Dv + k] : 0.0f; };
            Acc far_q = {}, far_k = {}, end = {};
            far_q = product(n, far_q, [&](int row, int k) { return grad_o(mine(row), k); }, of_s);
            far_k = product(n, far_k, [&](int row, int k) { return grad_v(mine(row), k); }, of_s);
            end = product(n, end, [&](int row, int k) { return u(mine(row), k); }, of_d);
            for (int r = 0; r < 4; ++r) {
                const int i = mine(group * 4 + r);
                const float f = gates.f[i], t = gates.t[i];
                const bool live = bit_of(alive, i);
                far_q[r] = f == 0.0f || !live ? 0.0f : p.scale * f * far_q[r];
                far_k[r] = f == 0.0f || !live ? 0.0f : -f * far_k[r];
                end[r] = t == 0.0f || !live ? 0.0f : t * end[r];
                if (t != 0.0f && live) at_end = fmaf(K[i * LD + d], end[r], at_end);
            }
            auto of_k = [&](int k, int c) { return K[k * LD + tile * 16 + c]; };
            auto of_q = [&](int k, int c) { return Q[k * LD + tile * 16 + c]; };
            auto n_row = [&](int row, int k) { return dN[mine(row) * LN + k]; };
            auto m_row = [&](int row, int k) { return dM[mine(row) * LN + k]; };
            auto n_col = [&](int row, int k) { return dN[k * LN + mine(row)]; };
            auto m_col = [&](int row, int k) { return dM[k * LN + mine(row)]; };
            if (bad) {
                auto before = [&](int row, int k) {
                    const int i = mine(row);
                    return k <= i && bit_of(alive, i) && bit_of(alive, k) && joined(starts, i, k);
                };
                auto behind = [&](int row, int k) {
                    const int i = mine(row);
                    return k >= i && bit_of(alive, i) && bit_of(alive, k) && joined(starts, k, i);
                };
                dq[tile] = careful_product(kSteps, far_q, n_row, of_k, before);
                plus[tile] = careful_product(kSteps, far_k, m_row, of_k, before);
                minus[tile] = careful_product(kSteps, end, n_col, of_q, behind);
                minus[tile] = careful_product(kSteps, minus[tile], m_col, of_k, behind);
            } else {
                dq[tile] = product(kSteps, far_q, n_row, of_k);
                plus[tile] = product(kSteps, far_k, m_row, of_k);
                minus[tile] = product(kSteps, end, n_col, of_q);
                minus[tile] = product(kSteps, minus[tile], m_col, of_k);
            }
            for (int r = 0; r < 4; ++r) {
                const int i = mine(group * 4 + r);
                dot[r] = fmaf(Q[i * LD + d], dq[tile][r], fmaf(K[i * LD + d], plus[tile][r] - minus[tile][r], dot[r]));
                sum_q[tile][r] += dq[tile][r];
                sum_k[tile][r] += plus[tile][r] + minus[tile][r];
            }
        }
        for (int r = 0; r < 4; ++r) {
            const float v = row_sum(dot[r]);
            if (at == 0) dG[mine(group * 4 + r)] = v;
        }
        const float whole = gates.f[kSteps - 1];
        if (whole != 0.0f) {
            float v = 0.0f;
            for (int e = threadIdx.x; e < p.Dk * p.Dv; e += kDeltaThreads) v = fmaf(D[e], S[e], v);
            at_end = fmaf(whole, v, at_end);
        }
        for (int d = 1; d < kWave; d *= 2) at_end += __shfl_xor(at_end, d);
        if (lane == 0) extra[wave] = at_end;
        __syncthreads();
        if (wave == 0) {
            const int i = lane, t = chunk * kSteps + i, part = part_of(starts, i);
            float v = dG[i];
            if (i == kSteps - 1) v += (extra[0] + extra[1]) + (extra[2] + extra[3]);
            double s = v;
            for (int d = 1; d < kWave; d *= 2) {
                const double later = __shfl_down(s, d);
                const int its = __shfl_down(part, d);
                if (i + d < kWave && its == part) s += later;
            }
            if (t < p.T) {
                const int64_t to = (b * p.T + t) * p.Hv + h;
                p.grad_log_decay[to] = bit_of(alive, i) && !bit_of(starts, i) ? (float)s : 0.0f;
                p.grad_beta[to] = bit_of(alive, i) ? dbeta[i] : 0.0f;
            }
        }
    }
#pragma unroll
    for (int tile = 0; tile < kTiles; ++tile)
        for (int r = 0; r < 4; ++r) {
            const int i = wave * 16 + group * 4 + r, t = chunk * kSteps + i, d = tile * 16 + at;
            if (t >= p.T || d >= p.Dk) continue;
            const bool live = bit_of(gates.live, i);
            const_cast<E *>(row_at<E>(p.grad_q, p.ld_gq, b, p.T, t, hk, p.Dk))[d] = from_f32<E>(live ? sum_q[tile][r] : 0.0f);
            const_cast<E *>(row_at<E>(p.grad_k, p.ld_gk, b, p.T, t, hk, p.Dk))[d] = from_f32<E>(live ? sum_k[tile][r] : 0.0f);
        }
}

template <typename E, int DK>
int run(const DeltaArgs &p, hipStream_t stream)
{
    size_t lds = (size_t)(2 * kSteps * (DK + 1) + kCols * (DK + 1) + 3 * kCols * (kSteps + 1)) * sizeof(float);
    if (const int rc = make_room_for(reinterpret_cast<const void *>(back_kernel<E, DK>), lds)) return rc;
    const int blocks = (p.Dv + kCols - 1) / kCols;
    hipLaunchKernelGGL((back_kernel<E, DK>), dim3((unsigned)((int64_t)p.B * p.Hv * blocks)), dim3(kDeltaThreads), lds, stream, p);
    if (p.chunks > 0) {
        lds = (size_t)(2 * kSteps * (DK + 1) + 2 * kSteps * (kSteps + 1)) * sizeof(float);
        if (const int rc = make_room_for(reinterpret_cast<const void *>(chunk_grad_kernel<E, DK>), lds)) return rc;
        hipLaunchKernelGGL((chunk_grad_kernel<E, DK>), dim3((unsigned)((int64_t)p.B * p.Hk * p.chunks)), dim3(kDeltaThreads), lds, stream, p);
    }
    return launched("delta scan gradient");
}

}  // namespace

int delta_grad_launch(int dtype, const DeltaArgs &p, hipStream_t stream)
{
    return with_dtype(dtype, [&](auto e) { return with_keys(p.Dk, [&](auto dk) { return run<decltype(e), decltype(dk)::value>(p, stream); }); });
}

}  // namespace marl
