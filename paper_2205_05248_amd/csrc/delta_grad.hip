// Gated delta rule, backward: the way back through the chunks, then the gradients of every chunk side by side.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "delta.h"

namespace marl {
namespace {

// The chunks of one head from the last to the first, for 16 NT value columns as in the forward pass: D, Y and the gradient of v.  Wave w has
// rows 16 w on of the chunk, and rows w DK / 4 on of the adjoint, which stays in its accumulators.
template <typename E, int DK, int NT>
__global__ __launch_bounds__(kDeltaThreads, NT == 1 && kExact<E> * DK <= 128 ? 2 : 1) void back_kernel(DeltaArgs p)
{
    constexpr int PE = kExact<E>, KS = DK / 32, LS = DK + 8, LU = kSteps + 8, C = 16 * NT;
    constexpr int kTiles = (DK + 63) / 64;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    typedef __bf16 StatePlane[C][LS];
    typedef __bf16 StepPlane[C][LU];
    StatePlane *S = reinterpret_cast<StatePlane *>(lds);                           // [3], columns of the adjoint
    // the upstream gradient of this chunk and of the next: [PE] as it is, [3] scaled by what of it reaches the state before
    StepPlane *upstream = reinterpret_cast<StepPlane *>(lds + 3 * sizeof(StatePlane)), *R = upstream + 2 * (PE + 3), *V = R + 3;      // [3], [3]
    __shared__ int not_finite[4];                      // upstream of even and odd chunks, beta dU, dV
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, at = lane % 16, group = lane / 16;
    const Place place = place_of((int64_t)p.B * p.Hv, p.Dv, C);
    if (place.head < 0) return;                        // the whole workgroup
    const int64_t head = place.head, b = head / p.Hv;
    const int col = place.first + at * NT, h = (int)(head % p.Hv), hk = h / (p.Hv / p.Hk);
    const int64_t key_head = b * p.Hk + hk;
    const bool has_state = wave * kTiles * 16 < DK;
    Acc adj[kTiles][NT] = {};
    if (p.grad_s_last && has_state)
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = (wave * kTiles + tile) * 16 + group * 4 + r;
                float v[NT] = {};
                if (d < p.Dk) read_columns<float, NT>(p.grad_s_last + (head * p.Dk + d) * p.Dv, col, p.Dv, v);
#pragma unroll
                for (int n = 0; n < NT; ++n) adj[tile][n][r] = v[n];
            }
    Frag k[KS][PE];
    float go[4][NT];
    Acc f_next, t_next, beta_next;
    auto load_start = [&](int chunk) {
        const Frag *K = p.K + (key_head * p.chunks + chunk) * key_frags(DK, PE);
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int n = 0; n < PE; ++n) k[s][n] = K[frag_at(wave, s, n, KS, PE)];
        const ChunkGates &g = p.gates[head * p.chunks + chunk];
        f_next = *reinterpret_cast<const Acc *>(g.f + wave * 16 + group * 4);
        t_next = *reinterpret_cast<const Acc *>(g.t + wave * 16 + group * 4);
        beta_next = *reinterpret_cast<const Acc *>(g.beta + wave * 16 + group * 4);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = chunk * kSteps + wave * 16 + group * 4 + r;
#pragma unroll
            for (int n = 0; n < NT; ++n) go[r][n] = 0.0f;
            if (t < p.T) read_columns<E, NT>(row_at<E>(p.grad_o, p.ld_go, b, p.T, t, h, p.Dv), col, p.Dv, go[r]);
        }
    };
    auto adjoint_out = [&](float *to) {                // [Dk,Dv]
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = (wave * kTiles + tile) * 16 + group * 4 + r;
                float v[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) v[n] = adj[tile][n][r];
                if (d < p.Dk) write_columns<float, NT>(to + (int64_t)d * p.Dv, col, p.Dv, v);
            }
    };
    auto share_adjoint = [&] {
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                Four planes[3];
                split(adj[tile][n], planes);
#pragma unroll
                for (int m = 0; m < 3; ++m) *reinterpret_cast<Four *>(&S[m][n * 16 + at][(wave * kTiles + tile) * 16 + group * 4]) = planes[m];
            }
    };
    auto share_steps = [&](StepPlane *to, auto &planes, int n) {
        constexpr int PLANES = sizeof(planes) / sizeof(Four);
#pragma unroll
        for (int m = 0; m < PLANES; ++m) *reinterpret_cast<Four *>(&to[m][n * 16 + at][wave * 16 + group * 4]) = planes[m];
    };
    auto share_upstream = [&](int chunk) {
        const unsigned long long live = p.gates[head * p.chunks + chunk].live;
        StepPlane *O = upstream + chunk % 2 * (PE + 3), *Of = O + PE;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            Acc o, of;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                o[r] = bit_of(live, wave * 16 + group * 4 + r) ? go[r][n] : 0.0f;
                of[r] = f_next[r] == 0.0f ? 0.0f : p.scale * f_next[r] * o[r];
            }
            Four exact[PE], planes[3];
            split(o, exact);
            split(of, planes);
            share_steps(O, exact, n);
            share_steps(Of, planes, n);
            if (!all_finite(o)) not_finite[chunk % 2] = 1;
        }
    };
    if (threadIdx.x < 4) not_finite[threadIdx.x] = 0;
    __syncthreads();
    if (p.chunks > 0) {
        load_start(p.chunks - 1);
        share_upstream(p.chunks - 1);
    }
    if (has_state) share_adjoint();
    __syncthreads();
    for (int chunk = p.chunks - 1; chunk >= 0; --chunk) {
        const int64_t record = head * p.chunks + chunk;
        const ChunkGates &g = p.gates[record];
        const unsigned long long starts = g.starts, live = g.live;
        const float whole = g.f[kSteps - 1];
        const bool bad = g.bad != 0, careful_o = bad || not_finite[chunk % 2];
        const StepPlane *O = upstream + chunk % 2 * (PE + 3), *Of = O + PE;
        // flags are taken back where all have read them and none sets them before the next barrier
        if (threadIdx.x == 0) not_finite[(chunk + 1) % 2] = not_finite[3] = 0;
        if (has_state) adjoint_out(p.D + record * p.Dk * p.Dv);
        Frag nn[2][3], pp[2][3], kt[kTiles][2][PE], qt[kTiles][2][PE];
        const Frag *N = p.NT + record * square_frags(3), *P = p.PT + record * square_frags(3);
        const Frag *KT = p.KT + (key_head * p.chunks + chunk) * key_frags(DK, PE), *QT = p.QT + (key_head * p.chunks + chunk) * key_frags(DK, PE);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (s * 32 + 31 < wave * 16) continue;     // zeros
#pragma unroll
            for (int n = 0; n < 3; ++n) {
                pp[s][n] = P[frag_at(wave, s, n, 2, 3)];
                nn[s][n] = N[frag_at(wave, s, n, 2, 3)];
            }
        }
        // dU = P' dO + t K D
        const Acc f = f_next, t = t_next, beta = beta_next;
        Acc y[NT] = {};
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                Frag of_state[3];
#pragma unroll
                for (int m = 0; m < 3; ++m) of_state[m] = *reinterpret_cast<const Frag *>(&S[m][n * 16 + at][s * 32 + group * 8]);
                y[n] = multiply<PE, 3>(k[s], of_state, y[n]);
            }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int r = 0; r < 4; ++r) y[n][r] = t[r] == 0.0f || !bit_of(live, wave * 16 + group * 4 + r) ? 0.0f : t[r] * y[n][r];
            if (careful_o) {
                unsigned long long pass[4];
                for (int r = 0; r < 4; ++r) {
                    const int i = wave * 16 + group * 4 + r;
                    pass[r] = bit_of(live, i) ? from(starts, i) & live : 0;
                }
                y[n] = careful_multiply(y[n], P, wave, 3, O[0][n * 16 + at], PE, C * LU, pass);
            } else {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    if (s * 32 + 31 < wave * 16) continue;
                    Frag of_o[PE];
#pragma unroll
                    for (int x = 0; x < PE; ++x) of_o[x] = *reinterpret_cast<const Frag *>(&O[x][n * 16 + at][s * 32 + group * 8]);
                    y[n] = multiply<3, PE>(pp[s], of_o, y[n]);
                }
            }
            const Acc minus = -(beta * y[n]);
            Four planes[3];
            split(minus, planes);
            share_steps(R, planes, n);
            if (!all_finite(minus)) not_finite[2] = 1;
        }
        __syncthreads();
        // Y = dU - N' (beta dU), dV = beta Y
        if (has_state)
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int n = 0; n < PE; ++n) {
                        kt[tile][s][n] = KT[frag_at(wave * kTiles + tile, s, n, 2, PE)];
                        qt[tile][s][n] = QT[frag_at(wave * kTiles + tile, s, n, 2, PE)];
                    }
        const bool careful_n = bad || not_finite[2];
        Acc v[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (careful_n) {
                unsigned long long pass[4];
                for (int r = 0; r < 4; ++r) {
                    const int i = wave * 16 + group * 4 + r;
                    pass[r] = bit_of(live, i) ? from(starts, i) & live & ~(1ull << i) : 0;
                }
                y[n] = careful_multiply(y[n], N, wave, 3, R[0][n * 16 + at], 3, C * LU, pass);
            } else {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    if (s * 32 + 31 < wave * 16) continue;
                    Frag of_r[3];
#pragma unroll
                    for (int x = 0; x < 3; ++x) of_r[x] = *reinterpret_cast<const Frag *>(&R[x][n * 16 + at][s * 32 + group * 8]);
                    y[n] = multiply<3, 3>(nn[s], of_r, y[n]);
                }
            }
            Acc back;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (!bit_of(live, wave * 16 + group * 4 + r)) y[n][r] = 0.0f;
                v[n][r] = beta[r] * y[n][r];
                back[r] = f[r] == 0.0f ? 0.0f : -f[r] * v[n][r];
            }
            Four planes[3];
            split(back, planes);
            share_steps(V, planes, n);
            if (!all_finite(v[n])) not_finite[3] = 1;
        }
        if (chunk > 0) load_start(chunk - 1);
        __syncthreads();
        // D <- f_63 D + (scale f Q)' dO - (f K)' dV
        if (has_state) {
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) adj[tile][n][r] = whole == 0.0f ? 0.0f : whole * adj[tile][n][r];
            if (careful_o || not_finite[3]) {
                unsigned long long pass[4];
                for (int r = 0; r < 4; ++r) pass[r] = (starts ? (starts & -starts) - 1 : ~0ull) & live;
                for (int tile = 0; tile < kTiles; ++tile)
                    for (int n = 0; n < NT; ++n) {
                        adj[tile][n] = careful_multiply(adj[tile][n], QT, wave * kTiles + tile, PE, Of[0][n * 16 + at], 3, C * LU, pass);
                        adj[tile][n] = careful_multiply(adj[tile][n], KT, wave * kTiles + tile, PE, V[0][n * 16 + at], 3, C * LU, pass);
                    }
            } else {
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        Frag of_o[3], of_v[3];
#pragma unroll
                        for (int x = 0; x < 3; ++x) {
                            of_o[x] = *reinterpret_cast<const Frag *>(&Of[x][n * 16 + at][s * 32 + group * 8]);
                            of_v[x] = *reinterpret_cast<const Frag *>(&V[x][n * 16 + at][s * 32 + group * 8]);
                        }
#pragma unroll
                        for (int tile = 0; tile < kTiles; ++tile) {
                            adj[tile][n] = multiply<PE, 3>(qt[tile][s], of_o, adj[tile][n]);
                            adj[tile][n] = multiply<PE, 3>(kt[tile][s], of_v, adj[tile][n]);
                        }
                    }
            }
            share_adjoint();
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = wave * 16 + group * 4 + r, step = chunk * kSteps + i;
            float x[NT], z[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) x[n] = y[n][r], z[n] = bit_of(live, i) ? v[n][r] : 0.0f;
            write_columns<float, NT>(p.Y + (record * kSteps + i) * p.Dv, col, p.Dv, x);
            if (step < p.T) write_columns<E, NT>(const_cast<E *>(row_at<E>(p.grad_v, p.ld_gv, b, p.T, step, h, p.Dv)), col, p.Dv, z);
        }
        if (chunk > 0) share_upstream(chunk - 1);
        if (threadIdx.x == 0) not_finite[2] = 0;
        __syncthreads();
    }
    if (p.grad_s_first && has_state) adjoint_out(p.grad_s_first + head * p.Dk * p.Dv);
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
    extern __shared__ __attribute__((aligned(16))) char lds[];
    float *K = reinterpret_cast<float *>(lds), *Q = K + kSteps * LD, *dN = Q + kSteps * LD, *dM = dN + kSteps * LN;
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

template <typename E, int DK, int NT>
int run_back(const DeltaArgs &p, hipStream_t stream)
{
    const size_t lds = (size_t)16 * NT * (3 * (DK + 8) + (12 + 2 * kExact<E>) * (kSteps + 8)) * sizeof(__bf16);
    if (const int rc = make_room_for(reinterpret_cast<const void *>(back_kernel<E, DK, NT>), lds)) return rc;
    hipLaunchKernelGGL((back_kernel<E, DK, NT>), dim3(places((int64_t)p.B * p.Hv, p.Dv, 16 * NT)), dim3(kDeltaThreads), lds, stream, p);
    return launched("delta scan gradient");
}

template <typename E, int DK>
int run(const DeltaArgs &p, hipStream_t stream)
{
    const int rc = (int64_t)p.B * p.Hv * ((p.Dv + 31) / 32) >= 256 ? run_back<E, DK, 2>(p, stream) : run_back<E, DK, 1>(p, stream);
    if (rc || p.chunks == 0) return rc;
    const size_t lds = (size_t)(2 * kSteps * (DK + 1) + 2 * kSteps * (kSteps + 1)) * sizeof(float);
    if (const int failed = make_room_for(reinterpret_cast<const void *>(chunk_grad_kernel<E, DK>), lds)) return failed;
    hipLaunchKernelGGL((chunk_grad_kernel<E, DK>), dim3((unsigned)((int64_t)p.B * p.Hk * p.chunks)), dim3(kDeltaThreads), lds, stream, p);
    return launched("delta scan gradient");
}

}  // namespace

int delta_grad_launch(int dtype, const DeltaArgs &p, hipStream_t stream)
{
    return with_dtype(dtype, [&](auto e) { return with_keys(p.Dk, [&](auto dk) { return run<decltype(e), decltype(dk)::value>(p, stream); }); });
}

}  // namespace marl
