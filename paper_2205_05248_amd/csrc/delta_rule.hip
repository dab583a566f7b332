// Gated delta rule: the entry points, and the single step.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "delta.h"

namespace marl {
namespace {

struct StepArgs {
    int n, Hk, Hv, Dk, Dv, slots, tiles, vectors;
    const void *q, *k, *v;
    int64_t ld_q, ld_k, ld_v;
    const float *log_decay, *beta;
    float scale;
    const int32_t *slot;
    const uint8_t *reset;
    const float *s_in;
    float *s_out;
    void *o;
    int64_t ld_o;
};

constexpr int kRowsHeld = 16;                          // state rows of a thread: 128 over at least eight groups of threads

// A workgroup has one sequence, one head and up to 32 vectors of V columns; `vectors` (a power of two) threads lie along the columns,
// the others along the rows.  The state is read once, into registers: with k.S and q.S of the state before,
//   u = beta (v - a k.S)      S <- a S + k u      o = scale (a q.S + (q.k) u).
// Bound by the states' bytes: 201 x 16 x 128 x 128, 421 MB, in 87 us, 4.8 TB/s, as a large copy (105 us with stores through the caches, which
// keep what no one reads again; loads past them too: 95).
template <typename E, int V>
__global__ __launch_bounds__(kDeltaThreads) void step_kernel(StepArgs p)
{
    typedef float Vec __attribute__((ext_vector_type(V)));
    __shared__ Vec part_k[kDeltaThreads / kWave][32], part_q[kDeltaThreads / kWave][32];
    __shared__ float part_kq[kDeltaThreads / kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int tile = blockIdx.x % p.tiles, h = (int)(blockIdx.x / p.tiles % p.Hv), seq = (int)(blockIdx.x / p.tiles / p.Hv);
    const int x = threadIdx.x % p.vectors, y = threadIdx.x / p.vectors, groups = kDeltaThreads / p.vectors;
    const int col = (tile * p.vectors + x) * V;
    const bool in = col < p.Dv;
    const int slot = p.slot ? min(max(p.slot[seq], 0), p.slots - 1) : seq;
    const int64_t state = ((int64_t)slot * p.Hv + h) * p.Dk * p.Dv + col;
    const E *q = static_cast<const E *>(p.q) + seq * p.ld_q + (int64_t)(h / (p.Hv / p.Hk)) * p.Dk;
    const E *k = static_cast<const E *>(p.k) + seq * p.ld_k + (int64_t)(h / (p.Hv / p.Hk)) * p.Dk;
    const float g = p.log_decay[(int64_t)seq * p.Hv + h], beta = p.beta[(int64_t)seq * p.Hv + h];
    const bool fresh = (p.reset && p.reset[seq]) || g == -__builtin_inff();
    const float a = decay_of(g < -200.0f ? -200.0 : (double)g);
    Vec held[kRowsHeld], ks = 0.0f, qs = 0.0f;
    float kd[kRowsHeld], kq = 0.0f;
#pragma unroll
    for (int r = 0; r < kRowsHeld; ++r) {
        const int d = r * groups + y;
        if (r * groups >= p.Dk) break;
        held[r] = in && d < p.Dk && !fresh ? *reinterpret_cast<const Vec *>(p.s_in + state + (int64_t)d * p.Dv) : (Vec)0.0f;
        kd[r] = d < p.Dk ? to_f32(k[d]) : 0.0f;
        const float qd = d < p.Dk ? to_f32(q[d]) : 0.0f;
        if (d < p.Dk) {
            ks += kd[r] * held[r];
            qs += qd * held[r];
            kq = fmaf(kd[r], qd, kq);
        }
    }
    for (int d = p.vectors; d < kWave; d *= 2) {
#pragma unroll
        for (int c = 0; c < V; ++c) {
            ks[c] += __shfl_xor(ks[c], d);
            qs[c] += __shfl_xor(qs[c], d);
        }
        kq += __shfl_xor(kq, d);
    }
    if (lane < p.vectors) {
        part_k[wave][lane] = ks;
        part_q[wave][lane] = qs;
    }
    if (lane == 0) part_kq[wave] = kq;
    __syncthreads();
    ks = part_k[0][x], qs = part_q[0][x], kq = part_kq[0];
#pragma unroll
    for (int w = 1; w < kDeltaThreads / kWave; ++w) ks += part_k[w][x], qs += part_q[w][x], kq += part_kq[w];
    if (!in) return;
    Vec u;
    const E *v = static_cast<const E *>(p.v) + seq * p.ld_v + (int64_t)h * p.Dv + col;
#pragma unroll
    for (int c = 0; c < V; ++c) u[c] = beta * (fresh ? to_f32(v[c]) : fmaf(-a, ks[c], to_f32(v[c])));
#pragma unroll
    for (int r = 0; r < kRowsHeld; ++r) {
        const int d = r * groups + y;
        if (r * groups >= p.Dk) break;
        if (d < p.Dk) __builtin_nontemporal_store(fresh ? kd[r] * u : a * held[r] + kd[r] * u, reinterpret_cast<Vec *>(p.s_out + state + (int64_t)d * p.Dv));
    }
    if (y == 0) {
        E *o = static_cast<E *>(p.o) + seq * p.ld_o + (int64_t)h * p.Dv + col;
#pragma unroll
        for (int c = 0; c < V; ++c) o[c] = from_f32<E>(p.scale * (fresh ? kq * u[c] : fmaf(a, qs[c], kq * u[c])));
    }
}

constexpr size_t up256(size_t n) { return (n + 255) / 256 * 256; }

struct Room { size_t gates, K, Q, KT, QT, N, P, NT, PT, S, M, D, Y, all; };
int planes_of(int dtype) { return dtype == MARL_DTYPE_F32 ? 3 : dtype == MARL_DTYPE_F16 ? 2 : 1; }
Room room_of(int dtype, const DeltaArgs &p, bool keep)
{
    const size_t records = (size_t)p.B * p.Hv * p.chunks, f = sizeof(float);
    const size_t keys = (size_t)p.B * p.Hk * p.chunks * key_frags(padded_keys(p.Dk), planes_of(dtype)) * sizeof(Frag);
    const size_t square = records * square_frags(3) * sizeof(Frag);
    Room r{};
    size_t at = 0;
    const auto take = [&](size_t bytes) { const size_t here = at; at += up256(bytes); return here; };
    r.gates = take(records * sizeof(ChunkGates));
    r.K = take(keys);
    r.Q = take(keys);
    r.KT = take(keys);
    r.N = take(square);
    r.P = take(square);
    if (keep) {
        r.QT = take(keys);
        r.NT = take(square);
        r.PT = take(square);
        const size_t state = records * padded_keys(p.Dk) * padded_values(p.Dv) * f, steps = records * kSteps * padded_values(p.Dv) * f;
        r.S = take(state);
        r.M = take(steps);
        r.D = take(state);
        r.Y = take(steps);
    }
    r.all = at;
    return r;
}
void place(int dtype, DeltaArgs &p, char *workspace, bool keep)
{
    const Room r = room_of(dtype, p, keep);
    const auto frags = [&](size_t at) { return reinterpret_cast<Frag *>(workspace + at); };
    const auto floats = [&](size_t at) { return reinterpret_cast<float *>(workspace + at); };
    p.gates = reinterpret_cast<ChunkGates *>(workspace + r.gates);
    p.K = frags(r.K); p.Q = frags(r.Q); p.KT = frags(r.KT); p.N = frags(r.N); p.P = frags(r.P);
    if (!keep) return;
    p.QT = frags(r.QT); p.NT = frags(r.NT); p.PT = frags(r.PT);
    p.S = floats(r.S); p.M = floats(r.M); p.D = floats(r.D); p.Y = floats(r.Y);
}

constexpr int64_t kMostRow = (int64_t)1 << 24;

int heads_check(int dtype, int Hk, int Hv, int Dk, int Dv)
{
    if (!known_dtype(dtype)) return MARL_ERR_BAD_DTYPE;
    if (Hk < 1 || Hv < Hk || Hv > 1024 || Hv % Hk != 0 || Dk < 1 || Dk > 128 || Dv < 1 || Dv > 1024) return MARL_ERR_BAD_DIM;
    return MARL_OK;
}
int sizes_check(int dtype, int B, int T, int Hk, int Hv, int Dk, int Dv)
{
    if (const int rc = heads_check(dtype, Hk, Hv, Dk, Dv)) return rc;
    if (B < 0 || T < 0 || (int64_t)B * Hv >= (1 << 24) || (int64_t)B * T >= (1 << 30)) return MARL_ERR_BAD_DIM;
    // a workgroup of up to 512 threads per record, and one of 256 per head and sixteen columns
    const int64_t heads = (int64_t)B * Hv;
    if (!fits_a_launch(heads * ((T + kSteps - 1) / kSteps), 512) || !fits_a_launch(heads * (padded_values(Dv) / 16) + 8, kDeltaThreads)) return MARL_ERR_BAD_DIM;
    return MARL_OK;
}
bool row_fits(int64_t ld, int H, int D) { return ld >= (int64_t)H * D && ld < kMostRow; }

DeltaArgs args_of(int B, int T, int Hk, int Hv, int Dk, int Dv, const void *q, int64_t ld_q, const void *k, int64_t ld_k, const void *v,
                  int64_t ld_v, const float *log_decay, const float *beta, float scale, const uint8_t *reset, const uint8_t *filled)
{
    DeltaArgs p{};
    p.B = B; p.T = T; p.Hk = Hk; p.Hv = Hv; p.Dk = Dk; p.Dv = Dv;
    p.chunks = (T + kSteps - 1) / kSteps;
    p.q = q; p.k = k; p.v = v; p.ld_q = ld_q; p.ld_k = ld_k; p.ld_v = ld_v;
    p.log_decay = log_decay; p.beta = beta; p.scale = scale; p.reset = reset; p.filled = filled;
    return p;
}

}  // namespace
}  // namespace marl

using namespace marl;

extern "C" {

int marl_delta_scan_workspace_bytes(int32_t dtype, int32_t B, int32_t T, int32_t Hk, int32_t Hv, int32_t Dk, int32_t Dv, int32_t keep,
                                    size_t *bytes)
{
    if (!bytes) return MARL_ERR_NULL;
    if (const int rc = sizes_check(dtype, B, T, Hk, Hv, Dk, Dv)) return rc;
    *bytes = room_of(dtype, args_of(B, T, Hk, Hv, Dk, Dv, nullptr, 0, nullptr, 0, nullptr, 0, nullptr, nullptr, 0, nullptr, nullptr), keep != 0).all;
    return MARL_OK;
}

int marl_delta_scan(int32_t dtype, int32_t B, int32_t T, int32_t Hk, int32_t Hv, int32_t Dk, int32_t Dv, const void *q, int64_t ld_q,
                    const void *k, int64_t ld_k, const void *v, int64_t ld_v, const float *log_decay, const float *beta, float scale,
                    const uint8_t *reset, const uint8_t *filled, const float *s_first, void *o, int64_t ld_o, float *s_last, int32_t keep,
                    void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (const int rc = sizes_check(dtype, B, T, Hk, Hv, Dk, Dv)) return rc;
    if (!std::isfinite(scale)) return MARL_ERR_BAD_ARG;
    if (B == 0) return MARL_OK;
    DeltaArgs p = args_of(B, T, Hk, Hv, Dk, Dv, q, ld_q, k, ld_k, v, ld_v, log_decay, beta, scale, reset, filled);
    const size_t need = room_of(dtype, p, keep != 0).all;
    if (T > 0) {
        if (!q || !k || !v || !log_decay || !beta || !o) return MARL_ERR_NULL;
        if (!row_fits(ld_q, Hk, Dk) || !row_fits(ld_k, Hk, Dk) || !row_fits(ld_v, Hv, Dv) || !row_fits(ld_o, Hv, Dv)) return MARL_ERR_BAD_DIM;
        if (o == q || o == k || o == v) return MARL_ERR_BAD_ARG;
        if (workspace_bytes < need) return MARL_ERR_BAD_DIM;
        if (!workspace) return MARL_ERR_NULL;
        if (!aligned_to(workspace, 256)) return MARL_ERR_BAD_ARG;
    }
    p.s_first = s_first; p.o = o; p.ld_o = ld_o; p.s_last = s_last;
    place(dtype, p, static_cast<char *>(workspace), keep != 0);
    return delta_scan_launch(dtype, p, static_cast<hipStream_t>(hip_stream));
}

int marl_delta_scan_grad(int32_t dtype, int32_t B, int32_t T, int32_t Hk, int32_t Hv, int32_t Dk, int32_t Dv, const void *q, int64_t ld_q,
                         const void *k, int64_t ld_k, const void *v, int64_t ld_v, const float *log_decay, const float *beta, float scale,
                         const uint8_t *reset, const uint8_t *filled, const void *grad_o, int64_t ld_go, const float *grad_s_last,
                         void *workspace, size_t workspace_bytes, void *grad_q, int64_t ld_gq, void *grad_k, int64_t ld_gk, void *grad_v,
                         int64_t ld_gv, float *grad_log_decay, float *grad_beta, float *grad_s_first, void *hip_stream)
{
    if (const int rc = sizes_check(dtype, B, T, Hk, Hv, Dk, Dv)) return rc;
    if (!std::isfinite(scale)) return MARL_ERR_BAD_ARG;
    if (B == 0) return MARL_OK;
    DeltaArgs p = args_of(B, T, Hk, Hv, Dk, Dv, q, ld_q, k, ld_k, v, ld_v, log_decay, beta, scale, reset, filled);
    if (T > 0) {
        if (!q || !k || !v || !log_decay || !beta || !grad_o || !grad_q || !grad_k || !grad_v || !grad_log_decay || !grad_beta) return MARL_ERR_NULL;
        if (!row_fits(ld_q, Hk, Dk) || !row_fits(ld_k, Hk, Dk) || !row_fits(ld_v, Hv, Dv) || !row_fits(ld_go, Hv, Dv) || !row_fits(ld_gq, Hk, Dk) ||
            !row_fits(ld_gk, Hk, Dk) || !row_fits(ld_gv, Hv, Dv))
            return MARL_ERR_BAD_DIM;
        for (const void *out : {grad_q, grad_k, grad_v})
            for (const void *in : {q, k, v, grad_o})
                if (out == in) return MARL_ERR_BAD_ARG;
        if (grad_q == grad_k || grad_q == grad_v || grad_k == grad_v) return MARL_ERR_BAD_ARG;
        if (workspace_bytes < room_of(dtype, p, true).all) return MARL_ERR_BAD_DIM;
        if (!workspace) return MARL_ERR_NULL;
        if (!aligned_to(workspace, 256)) return MARL_ERR_BAD_ARG;
    }
    p.grad_o = grad_o; p.ld_go = ld_go; p.grad_s_last = grad_s_last;
    p.grad_q = grad_q; p.grad_k = grad_k; p.grad_v = grad_v; p.ld_gq = ld_gq; p.ld_gk = ld_gk; p.ld_gv = ld_gv;
    p.grad_log_decay = grad_log_decay; p.grad_beta = grad_beta; p.grad_s_first = grad_s_first;
    place(dtype, p, static_cast<char *>(workspace), true);
    return delta_grad_launch(dtype, p, static_cast<hipStream_t>(hip_stream));
}

int marl_delta_step(int32_t dtype, int32_t n, int32_t Hk, int32_t Hv, int32_t Dk, int32_t Dv, const void *q, int64_t ld_q, const void *k,
                    int64_t ld_k, const void *v, int64_t ld_v, const float *log_decay, const float *beta, float scale, const int32_t *slot,
                    int32_t slots, const uint8_t *reset, const float *s_in, float *s_out, void *o, int64_t ld_o, void *hip_stream)
{
    if (const int rc = heads_check(dtype, Hk, Hv, Dk, Dv)) return rc;
    if (n < 0 || slots < 1 || (!slot && n > slots) || !fits_a_launch((int64_t)n * Hv * (padded_values(Dv) / 32), kDeltaThreads)) return MARL_ERR_BAD_DIM;
    if (!std::isfinite(scale)) return MARL_ERR_BAD_ARG;
    if (n == 0) return MARL_OK;
    if (!q || !k || !v || !log_decay || !beta || !s_in || !s_out || !o) return MARL_ERR_NULL;
    if (!row_fits(ld_q, Hk, Dk) || !row_fits(ld_k, Hk, Dk) || !row_fits(ld_v, Hv, Dv) || !row_fits(ld_o, Hv, Dv)) return MARL_ERR_BAD_DIM;
    if (o == q || o == k || o == v) return MARL_ERR_BAD_ARG;
    const bool fours = Dv % 4 == 0 && aligned_to(s_in, 16) && aligned_to(s_out, 16);
    const int all = fours ? Dv / 4 : Dv;
    int vectors = 1;
    while (vectors < 32 && vectors < all) vectors *= 2;
    const int tiles = (all + vectors - 1) / vectors;
    const StepArgs p{n, Hk, Hv, Dk, Dv, slots, tiles, vectors, q, k, v, ld_q, ld_k, ld_v, log_decay, beta, scale, slot, reset, s_in, s_out, o, ld_o};
    const dim3 grid((unsigned)((int64_t)n * Hv * tiles));
    return with_dtype(dtype, [&](auto e) {
        if (fours) hipLaunchKernelGGL((step_kernel<decltype(e), 4>), grid, dim3(kDeltaThreads), 0, static_cast<hipStream_t>(hip_stream), p);
        else hipLaunchKernelGGL((step_kernel<decltype(e), 1>), grid, dim3(kDeltaThreads), 0, static_cast<hipStream_t>(hip_stream), p);
        return launched("delta step");
    });
}

}  // extern "C"
