// Gated delta rule, forward: the matrices of every chunk side by side, then the way through the chunks.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "delta.h"

namespace marl {
namespace {

// Gates of a chunk, by one wave, a step a lane.
__device__ __forceinline__ void gates_of(const DeltaArgs &p, int64_t b, int h, int chunk, ChunkGates &out)
{
    const int i = threadIdx.x % kWave, t = chunk * kSteps + i;
    const int64_t step = b * p.T + t;
    const bool live = t < p.T && (!p.filled || p.filled[step]);
    float g = live ? p.log_decay[step * p.Hv + h] : 0.0f;
    const bool start = live && ((p.reset && p.reset[step]) || g == -__builtin_inff());
    g = start ? 0.0f : g < -200.0f ? -200.0f : g;
    const unsigned long long starts = __ballot(start);
    const unsigned long long upto = starts << (63 - i);
    const int first = upto ? i - __clzll((long long)upto) : 0;                     // of the lane's sequence
    double G = g;
    for (int d = 1; d < kWave; d *= 2) {
        const double before = __shfl_up(G, d);
        if (i - d >= first) G += before;
    }
    const int part = __popcll(upto);
    const double G_end = __shfl(G, 63);
    const int part_end = __shfl(part, 63);
    out.G[i] = G;
    out.f[i] = part == 0 ? decay_of(G) : 0.0f;
    out.t[i] = part == part_end ? decay_of(G_end - G) : 0.0f;
    out.beta[i] = live ? p.beta[step * p.Hv + h] : 0.0f;
    if (i == 0) out.starts = starts;
    const unsigned long long alive = __ballot(live);
    if (i == 0) { out.live = alive; out.bad = 0; }
}

// N and P of a chunk.  One workgroup; wave w has rows 16 w on.
template <typename E, int DK>
__global__ __launch_bounds__(kDeltaThreads) void chunk_kernel(DeltaArgs p)
{
    constexpr int LD = DK + 1, LN = kSteps + 1;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    float *K = lds, *Q = K + kSteps * LD, *A = Q + kSteps * LD, *N = A + kSteps * LN;
    __shared__ ChunkGates gates;
    __shared__ int bad;
    const int64_t record = blockIdx.x;
    const int chunk = (int)(record % p.chunks), h = (int)(record / p.chunks % p.Hv);
    const int64_t b = record / p.chunks / p.Hv;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, at = lane % 16, group = lane / 16;
    if (wave == 0) gates_of(p, b, h, chunk, gates);
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    const int hk = h / (p.Hv / p.Hk);
    for (int e = threadIdx.x; e < kSteps * DK; e += kDeltaThreads) {
        const int i = e / DK, d = e % DK;
        const bool is = bit_of(gates.live, i) && d < p.Dk;
        K[i * LD + d] = is ? to_f32(row_at<E>(p.k, p.ld_k, b, p.T, chunk * kSteps + i, hk, p.Dk)[d]) : 0.0f;
        Q[i * LD + d] = is ? to_f32(row_at<E>(p.q, p.ld_q, b, p.T, chunk * kSteps + i, hk, p.Dk)[d]) : 0.0f;
    }
    for (int e = threadIdx.x; e < kSteps * LN; e += kDeltaThreads) A[e] = N[e] = 0.0f;
    __syncthreads();
    float *P_out = p.P + record * kSteps * kSteps;
    bool fine = true;
    for (int tile = 0; tile < 4; ++tile) {
        Acc kk = {}, qk = {};
        if (tile <= wave) {
            auto keys = [&](int k, int col) { return K[(tile * 16 + col) * LD + k]; };
            kk = product(DK, kk, [&](int row, int k) { return K[(wave * 16 + row) * LD + k]; }, keys);
            qk = product(DK, qk, [&](int row, int k) { return Q[(wave * 16 + row) * LD + k]; }, keys);
        }
        const int j = tile * 16 + at;
        for (int r = 0; r < 4; ++r) {
            const int i = wave * 16 + group * 4 + r;
            const bool on = j <= i && bit_of(gates.live, i) && bit_of(gates.live, j) && joined(gates.starts, i, j);
            const float e = on ? decay_of(gates.G[i] - gates.G[j]) : 0.0f;
            const float a = on && j < i ? e * kk[r] : 0.0f, v = on ? p.scale * e * qk[r] : 0.0f;
            A[i * LN + j] = a;
            P_out[i * kSteps + j] = v;
            fine = fine && (a + v) * 0.0f == 0.0f;
        }
    }
    __syncthreads();
    // blocks on the diagonal: N_i = A_i - sum_j A_ij beta_j N_j, a column a lane
    {
        float n[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float v = A[(wave * 16 + i) * LN + wave * 16 + at];
#pragma unroll
            for (int j = 0; j < i; ++j) v = fmaf(-A[(wave * 16 + i) * LN + wave * 16 + j] * gates.beta[wave * 16 + j], n[j], v);
            n[i] = i > at ? v : 0.0f;
            if (group == 0) N[(wave * 16 + i) * LN + wave * 16 + at] = n[i];
            fine = fine && n[i] * 0.0f == 0.0f;
        }
    }
    __syncthreads();
    // block columns: N_ij = (I - N_ii beta) (A_ij - sum_m A_im beta_m N_mj), downwards
    for (int i = wave + 1; i < 4; ++i) {
        Acc c;
        for (int r = 0; r < 4; ++r) c[r] = A[(i * 16 + group * 4 + r) * LN + wave * 16 + at];
        c = product((i - wave) * 16, c, [&](int row, int k) { return -A[(i * 16 + row) * LN + wave * 16 + k] * gates.beta[wave * 16 + k]; },
                    [&](int k, int col) { return N[(wave * 16 + k) * LN + wave * 16 + col]; });
        for (int r = 0; r < 4; ++r) N[(i * 16 + group * 4 + r) * LN + wave * 16 + at] = c[r];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        c = product(16, c, [&](int row, int k) { return -N[(i * 16 + row) * LN + i * 16 + k] * gates.beta[i * 16 + k]; },
                    [&](int k, int col) { return N[(i * 16 + k) * LN + wave * 16 + col]; });
        __builtin_amdgcn_wave_barrier();
        for (int r = 0; r < 4; ++r) N[(i * 16 + group * 4 + r) * LN + wave * 16 + at] = c[r];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        fine = fine && all_finite(c);
    }
    if (!fine) bad = 1;
    __syncthreads();
    if (bad && wave == 0) {                            // again without anything that is not one of the sequence's steps in between
        for (int i = 0; i < kSteps; ++i) {
            float v = 0.0f;
            if (lane < i && joined(gates.starts, i, lane)) {
                v = A[i * LN + lane];
                for (int j = lane + 1; j < i; ++j)
                    if (bit_of(gates.live, j)) v = fmaf(-A[i * LN + j] * gates.beta[j], N[j * LN + lane], v);
            }
            N[i * LN + lane] = v;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
    __syncthreads();
    float *N_out = p.N + record * kSteps * kSteps;
    for (int e = threadIdx.x; e < kSteps * kSteps; e += kDeltaThreads) N_out[e] = N[e / kSteps * LN + e % kSteps];
    if (threadIdx.x == 0) gates.bad = bad;
    __syncthreads();
    const int *from = reinterpret_cast<const int *>(&gates);
    int *to = reinterpret_cast<int *>(p.gates + record);
    for (int e = threadIdx.x; e < (int)(sizeof(ChunkGates) / 4); e += kDeltaThreads) to[e] = from[e];
}

// The chunks of one head one after the other, for kCols value columns.  Wave w has rows 16 w on of the chunk, and rows
// w DK / 4 on of the state, which stays in its accumulators.
template <typename E, int DK>
__global__ __launch_bounds__(kDeltaThreads) void scan_kernel(DeltaArgs p)
{
    constexpr int LD = DK + 1, LS = DK + 1, LU = kSteps + 1;
    constexpr int kTiles = (DK + 63) / 64;             // of the state, for a wave; of DK = 32 two waves have one
    extern __shared__ __attribute__((aligned(16))) float lds[];
    float *K = lds, *Q = K + kSteps * LD, *S = Q + kSteps * LD, *R = S + kCols * LS, *U = R + kCols * LU, *Ue = U + kCols * LU;
    __shared__ ChunkGates gates;
    __shared__ int not_finite[2];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, at = lane % 16, group = lane / 16;
    const int blocks = (p.Dv + kCols - 1) / kCols;
    const int64_t head = blockIdx.x / blocks;
    const int first = (int)(blockIdx.x % blocks) * kCols, col = first + at;
    const int h = (int)(head % p.Hv), hk = h / (p.Hv / p.Hk);
    const int64_t b = head / p.Hv;
    const bool in = col < p.Dv;
    Acc state[kTiles];
    auto key_row = [&](int tile, int r) { return (wave * kTiles + tile) * 16 + group * 4 + r; };
#pragma unroll
    for (int tile = 0; tile < kTiles; ++tile)
        for (int r = 0; r < 4; ++r) {
            const int d = key_row(tile, r);
            state[tile][r] = p.s_first && in && d < p.Dk ? p.s_first[(head * p.Dk + d) * p.Dv + col] : 0.0f;
        }
    for (int chunk = 0; chunk < p.chunks; ++chunk) {
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
                if (d < DK) S[at * LS + d] = state[tile][r];
                if (p.S && in && d < p.Dk) p.S[(record * p.Dk + d) * p.Dv + col] = state[tile][r];
            }
        __syncthreads();
        for (int e = threadIdx.x; e < kSteps * DK; e += kDeltaThreads) {
            const int i = e / DK, d = e % DK;
            const bool is = bit_of(gates.live, i) && d < p.Dk;
            K[i * LD + d] = is ? to_f32(row_at<E>(p.k, p.ld_k, b, p.T, chunk * kSteps + i, hk, p.Dk)[d]) : 0.0f;
            Q[i * LD + d] = is ? to_f32(row_at<E>(p.q, p.ld_q, b, p.T, chunk * kSteps + i, hk, p.Dk)[d]) : 0.0f;
        }
        __syncthreads();
        auto of_state = [&](int k, int c) { return S[c * LS + k]; };
        Acc ks = {}, qs = {};
        ks = product(DK, ks, [&](int row, int k) { return K[(wave * 16 + row) * LD + k]; }, of_state);
        qs = product(DK, qs, [&](int row, int k) { return Q[(wave * 16 + row) * LD + k]; }, of_state);
        Acc m, scaled;
        for (int r = 0; r < 4; ++r) {
            const int i = wave * 16 + group * 4 + r;
            const bool live = bit_of(gates.live, i);
            const float v = live && in ? to_f32(row_at<E>(p.v, p.ld_v, b, p.T, chunk * kSteps + i, h, p.Dv)[col]) : 0.0f;
            const float f = gates.f[i];
            m[r] = live ? f == 0.0f ? v : fmaf(-f, ks[r], v) : 0.0f;
            scaled[r] = gates.beta[i] * m[r];
            R[at * LU + i] = scaled[r];
        }
        if (!all_finite(scaled)) not_finite[0] = 1;
        __syncthreads();
        const unsigned long long starts = gates.starts, alive = gates.live;
        const float *N = p.N + (record * kSteps + wave * 16) * kSteps, *P = p.P + (record * kSteps + wave * 16) * kSteps;
        auto of_r = [&](int k, int c) { return R[c * LU + k]; };
        auto of_n = [&](int row, int k) { return -N[row * kSteps + k]; };
        if (gates.bad || not_finite[0])
            m = careful_product(kSteps, m, of_n, of_r, [&](int row, int k) {
                const int i = wave * 16 + row;
                return k < i && bit_of(alive, i) && bit_of(alive, k) && joined(starts, i, k);
            });
        else m = product((wave + 1) * 16, m, of_n, of_r);
        for (int r = 0; r < 4; ++r) {
            const int i = wave * 16 + group * 4 + r;
            const float t = gates.t[i];
            scaled[r] = gates.beta[i] * m[r];
            U[at * LU + i] = scaled[r];
            Ue[at * LU + i] = t == 0.0f ? 0.0f : t * scaled[r];
            if (p.M && in) p.M[(record * kSteps + i) * p.Dv + col] = m[r];
        }
        if (!all_finite(scaled)) not_finite[1] = 1;
        __syncthreads();
        Acc o;
        for (int r = 0; r < 4; ++r) {
            const float f = gates.f[wave * 16 + group * 4 + r];
            o[r] = f == 0.0f ? 0.0f : p.scale * f * qs[r];
        }
        auto of_u = [&](int k, int c) { return U[c * LU + k]; };
        auto of_p = [&](int row, int k) { return P[row * kSteps + k]; };
        if (gates.bad || not_finite[1])
            o = careful_product(kSteps, o, of_p, of_u, [&](int row, int k) {
                const int i = wave * 16 + row;
                return k <= i && bit_of(alive, i) && bit_of(alive, k) && joined(starts, i, k);
            });
        else o = product((wave + 1) * 16, o, of_p, of_u);
        for (int r = 0; r < 4; ++r) {
            const int i = wave * 16 + group * 4 + r, t = chunk * kSteps + i;
            if (t < p.T && in) const_cast<E *>(row_at<E>(p.o, p.ld_o, b, p.T, t, h, p.Dv))[col] = from_f32<E>(bit_of(alive, i) ? o[r] : 0.0f);
        }
        const float whole = gates.f[kSteps - 1];
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile) {
            for (int r = 0; r < 4; ++r) state[tile][r] = whole == 0.0f ? 0.0f : whole * state[tile][r];
            const int d0 = (wave * kTiles + tile) * 16;
            if (d0 < DK)
                state[tile] = product(kSteps, state[tile], [&](int row, int k) { return gates.t[k] == 0.0f ? 0.0f : K[k * LD + d0 + row]; },
                                      [&](int k, int c) { return Ue[c * LU + k]; });
        }
    }
    if (p.s_last)
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile)
            for (int r = 0; r < 4; ++r) {
                const int d = key_row(tile, r);
                if (in && d < p.Dk) p.s_last[(head * p.Dk + d) * p.Dv + col] = state[tile][r];
            }
}

template <typename E, int DK>
int run(const DeltaArgs &p, hipStream_t stream)
{
    if (p.chunks > 0) {
        const size_t lds = (size_t)(2 * kSteps * (DK + 1) + 2 * kSteps * (kSteps + 1)) * sizeof(float);
        if (const int rc = make_room_for(reinterpret_cast<const void *>(chunk_kernel<E, DK>), lds)) return rc;
        hipLaunchKernelGGL((chunk_kernel<E, DK>), dim3((unsigned)((int64_t)p.B * p.Hv * p.chunks)), dim3(kDeltaThreads), lds, stream, p);
    }
    const size_t lds = (size_t)(2 * kSteps * (DK + 1) + kCols * (DK + 1) + 3 * kCols * (kSteps + 1)) * sizeof(float);
    if (const int rc = make_room_for(reinterpret_cast<const void *>(scan_kernel<E, DK>), lds)) return rc;
    const int blocks = (p.Dv + kCols - 1) / kCols;
    hipLaunchKernelGGL((scan_kernel<E, DK>), dim3((unsigned)((int64_t)p.B * p.Hv * blocks)), dim3(kDeltaThreads), lds, stream, p);
    return launched("delta scan");
}

}  // namespace

int delta_scan_launch(int dtype, const DeltaArgs &p, hipStream_t stream)
{
    return with_dtype(dtype, [&](auto e) { return with_keys(p.Dk, [&](auto dk) { return run<decltype(e), decltype(dk)::value>(p, stream); }); });
}

}  // namespace marl
