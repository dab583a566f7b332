// Gated delta rule, what its kernels share: arguments, the workspace, the gates of a chunk, products on the matrix pipe.
//
// A chunk is 64 steps.  With G the running sum of the log decays since its start or since the last sequence that starts in it,
//   E_ij = e^(G_i - G_j) for j <= i of one sequence, else 0      A_ij = E_ij k_i.k_j (j < i)      P_ij = scale E_ij q_i.k_j
//   f_i = e^(G_i) in the sequence that the chunk begins in, else 0;   t_j = e^(G_63 - G_j) in the one that it ends in, else 0
// and S the state before the chunk,
//   R = V - f K S     N = (I + A beta)^-1 A     M = R - N (beta R)     U = beta M
//   O = scale f Q S + P U        S <- f_63 S + K' (t U)
// Backward, with D the adjoint of the state after the chunk:
//   dU = P' dO + t K D      Y = dU - N' (beta dU)      dV = beta Y      dbeta = M.Y      D <- f_63 D + (scale f Q)' dO - (f K)' dV
// Strictly lower N alone is kept, never the inverse's unit diagonal, so that what a step keeps of itself is not rounded.
// Factors f, t and E that are not 0 by their sequence are at least the smallest normal number: a state that is infinite or
// NaN stays so however far it decays, and 0 says that a sequence starts in between, across which nothing is multiplied.
#pragma once
#include "operator_types.h"

namespace marl {

constexpr int kSteps = 64;                             // of a chunk
constexpr int kCols = 16;                              // value columns of a workgroup on the way through the chunks
constexpr int kDeltaThreads = 256;

typedef float Acc __attribute__((ext_vector_type(4)));

struct ChunkGates {
    double G[kSteps];
    float f[kSteps], t[kSteps], beta[kSteps];
    unsigned long long starts, live;                   // bit i: step i starts a sequence; is none of the padding
    int bad;                                           // N or P hold an infinity or NaN
    int pad[27];
};
static_assert(sizeof(ChunkGates) % 128 == 0, "records begin at lines");

struct DeltaArgs {
    int B, T, Hk, Hv, Dk, Dv, chunks;
    const void *q, *k, *v;
    int64_t ld_q, ld_k, ld_v;
    const float *log_decay, *beta;
    float scale;
    const uint8_t *reset, *filled;
    const float *s_first;
    void *o;
    int64_t ld_o;
    float *s_last;
    // backward
    const void *grad_o;
    int64_t ld_go;
    const float *grad_s_last;
    void *grad_q, *grad_k, *grad_v;
    int64_t ld_gq, ld_gk, ld_gv;
    float *grad_log_decay, *grad_beta, *grad_s_first;
    // workspace, one record per (b, value head, chunk)
    ChunkGates *gates;
    float *N, *P;                                      // [64,64]
    float *S, *M;                                      // [Dk,Dv] before the chunk, [64,Dv]; null without keep
    float *D, *Y;                                      // [Dk,Dv] adjoint behind the chunk, [64,Dv]
};

__device__ __forceinline__ float max_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }      // NaN stays
__device__ __forceinline__ float decay_of(double d) { return max_of(expf((float)d), 1.17549435e-38f); }

// Sequences of a chunk that have started up to and with step i.
__device__ __forceinline__ int part_of(unsigned long long starts, int i) { return __popcll(starts << (63 - i)); }
__device__ __forceinline__ bool bit_of(unsigned long long bits, int i) { return bits >> i & 1; }
// Whether step j hands anything to step i >= j.
__device__ __forceinline__ bool joined(unsigned long long starts, int i, int j) { return part_of(starts, i) == part_of(starts, j); }

// D = A B + C on 16 x 16 tiles in fp32: a(row, k), b(k, col) give one entry each; lane l holds rows l / 16 * 4 .. + 4 of column l % 16.
template <class FA, class FB>
__device__ __forceinline__ Acc product(int K, Acc c, FA &&a, FB &&b)
{
    const int lane = threadIdx.x % kWave, at = lane % 16, group = lane / 16;
    for (int k = 0; k < K; k += 4) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a(at, k + group), b(k + group, at), c, 0, 0, 0);
    return c;
}
// The same without the matrix pipe, for chunks that hold an infinity or NaN: only entries of which pass(row, k) holds take part.
template <class FA, class FB, class FP>
__device__ __noinline__ Acc careful_product(int K, Acc c, FA &&a, FB &&b, FP &&pass)
{
    const int lane = threadIdx.x % kWave, at = lane % 16, group = lane / 16;
    for (int r = 0; r < 4; ++r) {
        const int row = group * 4 + r;
        float v = c[r];
        for (int k = 0; k < K; ++k)
            if (pass(row, k)) v = fmaf(a(row, k), b(k, at), v);
        c[r] = v;
    }
    return c;
}
__device__ __forceinline__ bool all_finite(Acc a)
{
    const Acc z = a * 0.0f;
    return (z[0] + z[1]) + (z[2] + z[3]) == 0.0f;
}

// Row of the elements of step t of sequence b and head h.
template <typename E>
__device__ __forceinline__ const E *row_at(const void *base, int64_t ld, int64_t b, int T, int t, int h, int D)
{
    return static_cast<const E *>(base) + (b * T + t) * ld + (int64_t)h * D;
}

int delta_scan_launch(int dtype, const DeltaArgs &p, hipStream_t stream);
int delta_grad_launch(int dtype, const DeltaArgs &p, hipStream_t stream);

// Calls f with the padded key size as a constant.
template <typename F>
inline int with_keys(int Dk, F &&f)
{
    if (Dk <= 32) return f(std::integral_constant<int, 32>{});
    if (Dk <= 64) return f(std::integral_constant<int, 64>{});
    return f(std::integral_constant<int, 128>{});
}

// Shared memory beyond 64 KB has to be asked for.
inline int make_room_for(const void *kernel, size_t lds)
{
    if (lds <= 64 * 1024) return MARL_OK;
    const hipError_t err = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    return err == hipSuccess ? MARL_OK : report_device_error(err, "hipFuncSetAttribute");
}

}  // namespace marl
