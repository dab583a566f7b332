// Gated delta rule, backward: the way back through the chunks, then the gradients of every chunk side by side.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "delta.h"

namespace marl {
namespace {

// The chunks of one head from the last to the first, for 16 NT value columns as in the forward pass: D, Y and the gradient of v.  Wave w has
// rows 16 w on of the chunk, and rows w DK / 4 on of the adjoint, which stays in its accumulators.  Loads as in the forward pass, and bound by the
// same chain: 4 x 8192 x 16 heads x 128 x 128 bf16 700 us, 5.5 a chunk; the 320 x 120 batch with 4 heads of 16 in fp32 83.
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
    const int lane = threadIdx.x % kWave, wave = wave_index(), at = lane % 16, group = lane / 16, zero = hidden_zero();
    const Place place = place_of((int64_t)p.B * p.Hv, p.Dv, C);
    if (place.head < 0) return;                        // the whole workgroup
    const int64_t head = place.head, b = head / p.Hv;
    const int col = place.first + at * NT, h = (int)(head % p.Hv), hk = h / (p.Hv / p.Hk), DV = padded_values(p.Dv);
    const int64_t key_head = b * p.Hk + hk;
    const bool has_state = DK >= 64 || wave * 16 < DK;
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
    Frag k[KS][PE], n_of[2][3], p_of[2][3], kt[kTiles][2][PE], qt[kTiles][2][PE];
    Columns<E, NT> up[4];
    Acc f_next, t_next, beta_next, f_up, t_up;
    float whole_next;
    int bad_next;
    const unsigned of_row = (wave * 16 + group * 4) * 4u, row_bytes = (unsigned)p.ld_go * (unsigned)sizeof(E);
    const unsigned first_o = (wave * 16 + group * 4) * row_bytes + (unsigned)min(col, p.Dv - NT) * (unsigned)sizeof(E);
    auto load_start = [&](int chunk) {
        const ChunkGates *g = p.gates + head * p.chunks + chunk;
        const FragReader K(p.K + (key_head * p.chunks + chunk) * key_frags(DK, PE)), P(p.PT + (head * p.chunks + chunk) * square_frags(3));
        f_next = read_at<Acc>(g->f, of_row);
        t_next = read_at<Acc>(g->t, of_row);
        beta_next = read_at<Acc>(g->beta, of_row);
        whole_next = read_at<float>(&g->whole, (unsigned)zero);
        bad_next = read_at<int>(&g->bad, (unsigned)zero);
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int n = 0; n < PE; ++n) k[s][n] = K.at(wave, s, n, KS, PE);
#pragma unroll
        for (int s = 0; s < 2; ++s)                    // (what lies on the other side of the diagonal is never written, and not used)
#pragma unroll
            for (int n = 0; n < 3; ++n) p_of[s][n] = P.at(wave, s, n, 2, 3);
    };
    auto load_n = [&](int chunk) {
        const FragReader N(p.NT + (head * p.chunks + chunk) * square_frags(3));
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int n = 0; n < 3; ++n) n_of[s][n] = N.at(wave, s, n, 2, 3);
    };
    auto load_end = [&](int chunk) {
        const int64_t key_record = key_head * p.chunks + chunk;
        const FragReader KT(p.KT + key_record * key_frags(DK, PE)), QT(p.QT + key_record * key_frags(DK, PE));
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int n = 0; n < PE; ++n) {
                    kt[tile][s][n] = KT.at((wave * kTiles + tile) % (DK / 16), s, n, 2, PE);
                    qt[tile][s][n] = QT.at((wave * kTiles + tile) % (DK / 16), s, n, 2, PE);
                }
    };
    auto load_upstream = [&](int chunk) {
        const ChunkGates *g = p.gates + head * p.chunks + chunk;
        f_up = read_at<Acc>(g->f, of_row);
        t_up = read_at<Acc>(g->t, of_row);
        const E *rows = row_at<E>(p.grad_o, p.ld_go, b, p.T, chunk * kSteps, h, p.Dv);
        const int last = p.T - chunk * kSteps;         // rows behind it are not read: the first one is instead
#pragma unroll
        for (int r = 0; r < 4; ++r) up[r].load(rows, wave * 16 + group * 4 + r < last ? first_o + r * row_bytes : first_o - (wave * 16 + group * 4) * row_bytes);
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
    auto steps_frag = [&](const StepPlane *from, int n, int s, auto &to) {
        constexpr int PLANES = sizeof(to) / sizeof(Frag);
#pragma unroll
        for (int m = 0; m < PLANES; ++m) to[m] = *reinterpret_cast<const Frag *>(&from[m][n * 16 + at][s * 32 + group * 8]);
    };
    auto share_upstream = [&](int chunk) {
        StepPlane *O = upstream + chunk % 2 * (PE + 3), *Of = O + PE;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            Acc o, of;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                o[r] = t_up[r] < 0.0f ? 0.0f : up[r].at(n, col, p.Dv);
                of[r] = f_up[r] == 0.0f ? 0.0f : p.scale * f_up[r] * o[r];
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
        load_upstream(p.chunks - 1);
        load_start(p.chunks - 1);
        load_n(p.chunks - 1);
        load_end(p.chunks - 1);
        share_upstream(p.chunks - 1);
        load_upstream(max(p.chunks - 2, 0));
    }
    if (has_state) share_adjoint();
    __syncthreads();
    for (int chunk = p.chunks - 1; chunk >= 0; --chunk) {
        const int64_t record = head * p.chunks + chunk;
        const int next = max(chunk - 1, 0);
        const Acc f = f_next, t = t_next, beta = beta_next;
        const float whole = whole_next;
        const StepPlane *O = upstream + chunk % 2 * (PE + 3), *Of = O + PE;
        const bool bad = __builtin_amdgcn_readfirstlane(bad_next) != 0;
        // dU = P' dO + t K D
        Frag of_o[2][NT][PE];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n) steps_frag(O, n, s, of_o[s][n]);
        const bool careful_o = bad || not_finite[chunk % 2];
        // flags are taken back where all have read them and none sets them before the next barrier
        if (threadIdx.x == 0) not_finite[(chunk + 1) % 2] = not_finite[3] = 0;
        Sums<2> kd[NT];
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                Frag of_state[3];
#pragma unroll
                for (int m = 0; m < 3; ++m) of_state[m] = *reinterpret_cast<const Frag *>(&S[m][n * 16 + at][s * 32 + group * 8]);
                multiply_into(kd[n], k[s], of_state);
            }
        Acc y[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const Acc of_k = total(kd[n]);
#pragma unroll
            for (int r = 0; r < 4; ++r) y[n][r] = t[r] > 0.0f || t[r] != t[r] ? t[r] * of_k[r] : 0.0f;
        }
        if (careful_o) {
            const unsigned long long starts = p.gates[record].starts, live = p.gates[record].live;
            unsigned long long pass[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = wave * 16 + group * 4 + r;
                pass[r] = bit_of(live, i) ? from(starts, i) & live : 0;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) y[n] = careful_multiply<3, PE>(y[n], p.PT + record * square_frags(3), wave, O[0][n * 16 + at], C * LU, pass);
        } else {
            Sums<2> po[NT];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (s * 32 + 31 < wave * 16) continue;
#pragma unroll
                for (int n = 0; n < NT; ++n) multiply_into(po[n], p_of[s], of_o[s][n]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) y[n] += total(po[n]);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const Acc minus = -(beta * y[n]);
            Four planes[3];
            split(minus, planes);
            share_steps(R, planes, n);
            if (!all_finite(minus)) not_finite[2] = 1;
        }
        load_start(next);
        if (has_state) {
            float *to = p.D + record * DK * DV;
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float c[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) c[n] = adj[tile][n][r];
                    write_columns<float, NT>(to, ((wave * kTiles + tile) * 16 + group * 4 + r) * DV + col, DK * DV, c);
                }
        }
        __syncthreads();
        // Y = dU - N' (beta dU), dV = beta Y
        Frag of_r[2][NT][3];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n) steps_frag(R, n, s, of_r[s][n]);
        if (bad || not_finite[2]) {
            const unsigned long long starts = p.gates[record].starts, live = p.gates[record].live;
            unsigned long long pass[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = wave * 16 + group * 4 + r;
                pass[r] = bit_of(live, i) ? from(starts, i) & live & ~(1ull << i) : 0;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) y[n] = careful_multiply<3, 3>(y[n], p.NT + record * square_frags(3), wave, R[0][n * 16 + at], C * LU, pass);
        } else {
            Sums<2> nr[NT];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (s * 32 + 31 < wave * 16) continue;
#pragma unroll
                for (int n = 0; n < NT; ++n) multiply_into(nr[n], n_of[s], of_r[s][n]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) y[n] += total(nr[n]);
        }
        Acc v[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            Acc back;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                y[n][r] = t[r] < 0.0f ? 0.0f : y[n][r];
                v[n][r] = t[r] < 0.0f ? 0.0f : beta[r] * y[n][r];
                back[r] = f[r] == 0.0f ? 0.0f : -f[r] * v[n][r];
            }
            Four planes[3];
            split(back, planes);
            share_steps(V, planes, n);
            if (!all_finite(v[n])) not_finite[3] = 1;
        }
        load_n(next);
        {
            const RowsOut<E, NT> out(p, p.grad_v, p.ld_gv, b, chunk, h);
            float *to = p.Y + record * kSteps * DV;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = wave * 16 + group * 4 + r;
                float c[NT], z[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) c[n] = y[n][r], z[n] = v[n][r];
                write_columns<float, NT>(to, i * DV + col, kSteps * DV, c);
                out.put(i, col, z);
            }
        }
        __syncthreads();
        // D <- f_63 D + (scale f Q)' dO - (f K)' dV
        if (has_state) {
            Frag of_f[2][NT][3], of_v[2][NT][3];
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    steps_frag(Of, n, s, of_f[s][n]);
                    steps_frag(V, n, s, of_v[s][n]);
                }
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) adj[tile][n][r] = whole == 0.0f ? 0.0f : whole * adj[tile][n][r];
            if (careful_o || not_finite[3]) {
                const unsigned long long starts = p.gates[record].starts, live = p.gates[record].live;
                const int64_t key_record = key_head * p.chunks + chunk;
                unsigned long long pass[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) pass[r] = (starts ? (starts & -starts) - 1 : ~0ull) & live;
#pragma unroll
                for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        adj[tile][n] = careful_multiply<PE, 3>(adj[tile][n], p.QT + key_record * key_frags(DK, PE), wave * kTiles + tile, Of[0][n * 16 + at], C * LU, pass);
                        adj[tile][n] = careful_multiply<PE, 3>(adj[tile][n], p.KT + key_record * key_frags(DK, PE), wave * kTiles + tile, V[0][n * 16 + at], C * LU, pass);
                    }
            } else {
                Sums<2> of_keys[kTiles][NT];
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int tile = 0; tile < kTiles; ++tile) {
                            multiply_into(of_keys[tile][n], qt[tile][s], of_f[s][n]);
                            multiply_into(of_keys[tile][n], kt[tile][s], of_v[s][n]);
                        }
#pragma unroll
                for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
                    for (int n = 0; n < NT; ++n) adj[tile][n] += total(of_keys[tile][n]);
            }
            share_adjoint();
        }
        load_end(next);
        if (chunk > 0) share_upstream(chunk - 1);
        load_upstream(max(chunk - 2, 0));
        if (threadIdx.x == 0) not_finite[2] = 0;
        __syncthreads();
    }
    if (p.grad_s_first && has_state)
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = (wave * kTiles + tile) * 16 + group * 4 + r;
                float v[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) v[n] = adj[tile][n][r];
                if (d < p.Dk) write_columns<float, NT>(p.grad_s_first + (head * p.Dk + d) * p.Dv, col, p.Dv, v);
            }
}

// Among the 16 lanes that hold a row: the value N lanes before, 0 before the first; the last one's; the sum.
template <int CONTROL>
__device__ __forceinline__ float of_row(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CONTROL, 0xf, 0xf, true)); }
template <int N> __device__ __forceinline__ float lanes_before(float v) { return of_row<0x110 + N>(v); }
__device__ __forceinline__ float last_lane(float v) { return of_row<0x15f>(v); }
__device__ __forceinline__ float row_sum(float v)
{
    v += of_row<0x128>(v);                             // rotations by 8, 4, 2 and 1
    v += of_row<0x124>(v);
    v += of_row<0x122>(v);
    return v + of_row<0x121>(v);
}

// A chunk's steps as planes in shared memory, rows of COLUMNS entries.
template <int COLUMNS> struct Rows { typedef __bf16 Plane[kSteps][COLUMNS + 8]; };
typedef Rows<kSteps>::Plane Plane;

template <int PLANES, class PLANE>
__device__ __forceinline__ void put_row(PLANE *to, int row, int col, const float *v)
{
    Frag f[PLANES];
    split(v, f);
#pragma unroll
    for (int n = 0; n < PLANES; ++n) *reinterpret_cast<Frag *>(&to[n][row][col]) = f[n];
}
template <int PLANES, class PLANE>
__device__ __forceinline__ void get_frag(const PLANE *from, int tile, int step, Frag (&to)[PLANES])
{
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int n = 0; n < PLANES; ++n) to[n] = *reinterpret_cast<const Frag *>(&from[n][tile * 16 + lane % 16][step * 32 + lane / 16 * 8]);
}

// c + a b over 64 columns k for chunks that hold an infinity or NaN: only the k in pass[r] take part in the lane's r-th row.  a: rows of tile
// `tile` in three planes; b: fragments of the transposed factor.
template <int PB>
__device__ __forceinline__ Acc careful_rows(Acc c, const Plane *a, int tile, const Frag *b, int b_tile, const unsigned long long (&pass)[4])
{
    const int lane = threadIdx.x % kWave, at = lane % 16, group = lane / 16;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int row = tile * 16 + group * 4 + r;
        float v = c[r];
#pragma unroll 1
        for (int k = 0; k < kSteps; ++k) {
            if (!bit_of(pass[r], k)) continue;
            float x = 0.0f, y = 0.0f;
            for (int n = 2; n >= 0; --n) x += (float)a[n][row][k];
            for (int n = PB - 1; n >= 0; --n)
                y += (float)reinterpret_cast<const __bf16 *>(b)[(((b_tile * 2 + k / 32) * PB + n) * kWave + at + k % 32 / 8 * 16) * 8 + k % 8];
            v = fmaf(x, y, v);
        }
        c[r] = v;
    }
    return c;
}

// Gradients of q, k, beta and the log decay of a chunk, the value heads of a key head one after the other.  With dP = scale dO U',
// dA = -(dV) U', their products dN and dM with E, and X = dM + dM':
//   dq = dN K + scale f dO S'      dk = dN' Q + X K - f dV S' + t U D'
// The log decay of a step has a part in everything that is handed on across it, and its gradient is the sum of that:
//   dg_i = sum_(m >= i > j) F_mj + sum_(m >= i) (q_m.(scale f dO S')_m - k_m.(f dV S')_m) + sum_(j < i) k_j.(t U D')_j + f_63 <D, S>
// with F_mj = dM_mj k_m.k_j + dN_mj q_m.k_j.  (A running sum of the differences of neighbours, sum_j F_ij - sum_j F_ji and so on, holds what does not cross i
// too, which has to cancel: at a decay of e^-12 a tenth of the gradient was rounding.)
// Value columns come 32 or 64 at a time through shared memory.  Products with rows and columns of steps are split over the waves by
// rows, those with key columns by columns (16 w on), so that every entry of S and D is split into planes once.
// Waves of a workgroup: with 128 keys eight, of which four form dP and four dA, else four that form both (1.64 -> 1.21 ms of 4 x 8192 x 16 heads x 128 x
// 128 bf16).  There it reads 2.9 GB and writes 0.4 in 1.16 ms, and waits 62 % of its waves' cycles: a workgroup of 512 threads with 256 registers each fills a
// compute unit, so that nothing else works while it waits for a block of columns.
constexpr int grad_waves(int DK) { return DK == 128 ? 8 : 4; }
constexpr int grad_columns(int DK) { return DK == 128 ? 64 : 32; }       // at a time: more do not fit the registers of four waves

template <typename E, int DK>
__global__ __launch_bounds__(grad_waves(DK) * kWave, 2) void chunk_grad_kernel(DeltaArgs p)
{
    constexpr int PE = kExact<E>, KS = DK / 32, kOrder = PE == 1 ? 0 : 2, kWaves = grad_waves(DK), kThreads = kWaves * kWave;
    constexpr int CB = grad_columns(DK);
    extern __shared__ __attribute__((aligned(16))) char lds[];
    typedef typename Rows<CB>::Plane Block;
    Block *U = reinterpret_cast<Block *>(lds), *V = U + 3, *O = V + 3;             // [3], [3], [PE]
    Plane *dN = reinterpret_cast<Plane *>(lds), *dNT = dN + 3, *X = dN;            // later in the same room, [3] each
    __shared__ ChunkGates gates;
    __shared__ int not_finite;
    __shared__ float far_of[kWaves][kSteps], later_of[kWaves][kSteps], crossing[8][kSteps], extra[kWaves], dbeta[kSteps];
    const int lane = threadIdx.x % kWave;
    int wave = wave_index(), at = lane % 16, group = lane / 16;
    int nothing;
    const int hk = (int)(blockIdx.x / p.chunks % p.Hk);
    int chunk = (int)(blockIdx.x % p.chunks);
    const int64_t b = blockIdx.x / p.chunks / p.Hk;
    const int shared = p.Hv / p.Hk, DV = padded_values(p.Dv);
    const bool has_keys = wave * 16 < DK;
    const Frag *K = p.K + (int64_t)blockIdx.x * key_frags(DK, PE), *Q = p.Q + (int64_t)blockIdx.x * key_frags(DK, PE);
    const Frag *KT = p.KT + (int64_t)blockIdx.x * key_frags(DK, PE), *QT = p.QT + (int64_t)blockIdx.x * key_frags(DK, PE);
    Acc sum_q[4] = {}, sum_k[4] = {};
    unsigned long long alive = 0;
    for (int member = 0; member < shared; ++member) {
        // else addresses, masks and the products of K and Q are formed before the loop, and 500 registers do not hold them
        nothing = hidden_zero();
        at += nothing;
        group += nothing;
        nothing = __builtin_amdgcn_readfirstlane(nothing);
        chunk += nothing;
        wave += nothing;
        K += nothing;
        Q += nothing;
        KT += nothing;
        QT += nothing;
        const int h = hk * shared + member;
        const int64_t record = (b * p.Hv + h) * p.chunks + chunk;
        const float *M = p.M + record * kSteps * DV, *Y = p.Y + record * kSteps * DV;
        const float *S = p.S + record * DK * DV, *D = p.D + record * DK * DV;
        Acc d_of[2][4] = {}, far_q[4] = {}, far_k[4] = {}, end[4] = {};            // d_of: dP, dA
        float dot_states = 0.0f, dot_beta = 0.0f;
        // A block of columns: S and D of the wave's keys, and eight columns at a time of M, Y and dO of the thread's step.  All loads go out
        // before any wait, those of the first block before the one for the gates.
        typedef float Eight __attribute__((ext_vector_type(8)));
        constexpr int kSteps32 = CB / 32, kPer = kThreads / kSteps, kHalves = CB / 8 / kPer;      // threads of a step, and how often eight columns each
        static_assert(kHalves >= 1, "every thread has columns");
        const int own = threadIdx.x / kPer;
        Eight s[kSteps32], d[kSteps32], m[kHalves], y[kHalves];
        float o[kHalves][8];
        const E *grad_o = row_at<E>(p.grad_o, p.ld_go, b, p.T, min(chunk * kSteps + own, p.T - 1), h, p.Dv);
        auto load = [&](int c0) {
#pragma unroll
            for (int step = 0; step < kSteps32; ++step) {
                const int from = (wave * 16 % DK + at) * DV + min(c0 + step * 32, DV - 32) + group * 8;
                s[step] = *reinterpret_cast<const Eight *>(S + from);
                d[step] = *reinterpret_cast<const Eight *>(D + from);
            }
#pragma unroll
            for (int half = 0; half < kHalves; ++half) {
                const int c = c0 + (threadIdx.x % kPer * kHalves + half) * 8, from = own * DV + min(c, DV - 8);
                m[half] = *reinterpret_cast<const Eight *>(M + from);
                y[half] = *reinterpret_cast<const Eight *>(Y + from);
#pragma unroll
                for (int e = 0; e < 8; ++e) o[half][e] = 0.0f;
                read_columns<E, 8>(grad_o, c, p.Dv, o[half]);
            }
        };
        constexpr int kWords = (int)(sizeof(ChunkGates) / 4), kTurns = (kWords + kThreads - 1) / kThreads;
        int words[kTurns];
#pragma unroll
        for (int e = 0; e < kTurns; ++e) words[e] = reinterpret_cast<const int *>(p.gates + record)[min(e * kThreads + (int)threadIdx.x, kWords - 1)];
        load(0);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kTurns; ++e)
            if (e * kThreads + (int)threadIdx.x < kWords) reinterpret_cast<int *>(&gates)[e * kThreads + threadIdx.x] = words[e];
        if (threadIdx.x == 0) not_finite = 0;
        __syncthreads();
        const unsigned long long starts = gates.starts;
        alive = gates.live;
        for (int c0 = 0; c0 < p.Dv; c0 += CB) {
            const int steps = min(kSteps32, (DV - c0) / 32);
            if (c0 > 0) load(c0);
            {
                const bool live = bit_of(alive, own);
                const float beta = gates.beta[own];
#pragma unroll
                for (int half = 0; half < kHalves; ++half) {
                    const int c = (threadIdx.x % kPer * kHalves + half) * 8;
                    const bool in = live && c < 32 * steps;
                    float u[8], v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        dot_beta = in ? fmaf(m[half][e], y[half][e], dot_beta) : dot_beta;
                        u[e] = in ? beta * m[half][e] : 0.0f;
                        v[e] = in ? beta * y[half][e] : 0.0f;
                        o[half][e] = in ? o[half][e] : 0.0f;
                    }
                    put_row<3>(U, own, c, u);
                    put_row<3>(V, own, c, v);
                    put_row<PE>(O, own, c, o[half]);
                }
            }
            __syncthreads();
#pragma unroll
            for (int step = 0; step < kSteps32; ++step) {
                if (step >= steps) continue;
                {
                    const int row = wave % 4;
                    Frag o[PE], v[3];
                    if (kWaves == 4 || wave < 4) get_frag(O, row, step, o);
                    if (kWaves == 4 || wave >= 4) get_frag(V, row, step, v);
#pragma unroll
                    for (int tile = 0; tile < 4; ++tile) {
                        if (tile > row) continue;
                        Frag u[3];
                        get_frag(U, tile, step, u);
                        if (kWaves == 4 || wave < 4) d_of[0][tile] = multiply<PE, 3>(o, u, d_of[0][tile]);
                        if (kWaves == 4) d_of[1][tile] = multiply<3, 3>(v, u, d_of[1][tile]);
                        else if (wave >= 4) d_of[0][tile] = multiply<3, 3>(v, u, d_of[0][tile]);
                    }
                }
                if (!has_keys) continue;
                Frag of_s[3], of_d[3];
#pragma unroll
                for (int e = 0; e < 8; ++e) dot_states = fmaf(s[step][e], d[step][e], dot_states);
                split(reinterpret_cast<const float *>(&s[step]), of_s);
                split(reinterpret_cast<const float *>(&d[step]), of_d);
#pragma unroll
                for (int row = 0; row < 4; ++row) {
                    __builtin_amdgcn_sched_barrier(0); // (loads of all rows at once would not fit the registers)
                    Frag o[PE], v[3], u[3];
                    get_frag(O, row, step, o);
                    get_frag(V, row, step, v);
                    get_frag(U, row, step, u);
                    far_q[row] = multiply<PE, 3>(o, of_s, far_q[row]);
                    far_k[row] = multiply<3, 3>(v, of_s, far_k[row]);
                    end[row] = multiply<3, 3>(u, of_d, end[row]);
                }
            }
            __syncthreads();
        }
        // what goes from step j to step i, and what of F crosses a step
        Acc dm[4];
        bool fine = true;
        unsigned long long before[4];                  // steps that hand something to the lane's rows
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = wave % 4 * 16 + group * 4 + r;
            before[r] = bit_of(alive, i) ? upto(starts, i) & alive : 0;
        }
        auto flows = [&](Acc (&of)[4], bool is_p) {    // of P, or of A
            const int row = wave % 4;
            Acc raw[4] = {};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                Frag mine[PE];
#pragma unroll
                for (int n = 0; n < PE; ++n) mine[n] = FragReader(is_p ? Q : K).at(row, s, n, KS, PE);
#pragma unroll
                for (int tile = 0; tile < 4; ++tile) {
                    if (tile > row) continue;
                    Frag other[PE];
#pragma unroll
                    for (int n = 0; n < PE; ++n) other[n] = FragReader(K).at(tile, s, n, KS, PE);
                    raw[tile] = multiply<PE, PE, kOrder>(mine, other, raw[tile]);
                }
            }
            float left[4] = {};                        // sums of the rows in the tiles before
#pragma unroll
            for (int tile = 0; tile < 4; ++tile) {
                const int j = tile * 16 + at;
                Acc d;
                float across = 0.0f;                   // from before j to j or later
                if (tile <= row)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int i = row * 16 + group * 4 + r;
                        const bool on = bit_of(before[r], j) && (is_p || j < i);
                        const float e = decay_of(gates.G[i] - gates.G[j]), v = (is_p ? p.scale : -1.0f) * e * of[tile][r];
                        d[r] = on ? v : 0.0f;
                        float sum = on ? v * raw[tile][r] : 0.0f;
                        sum += lanes_before<1>(sum);
                        sum += lanes_before<2>(sum);
                        sum += lanes_before<4>(sum);
                        sum += lanes_before<8>(sum);
                        const float before_j = left[r] + lanes_before<1>(sum);
                        across += j <= i ? before_j : 0.0f;
                        left[r] += last_lane(sum);
                    }
                else d = Acc{};
                fine = fine && all_finite(d);
                if (is_p) {
                    Four planes[3];
                    split(d, planes);
#pragma unroll
                    for (int n = 0; n < 3; ++n) {
                        *reinterpret_cast<Four *>(&dNT[n][j][row * 16 + group * 4]) = planes[n];
#pragma unroll
                        for (int r = 0; r < 4; ++r) dN[n][row * 16 + group * 4 + r][j] = planes[n][r];
                    }
                } else {
                    dm[tile] = d;
                }
                across += __shfl_xor(across, 16);
                across += __shfl_xor(across, 32);
                if (group == 0) crossing[(is_p ? 0 : 4) + row][j] = across;
            }
        };
        if constexpr (kWaves == 4) {
            flows(d_of[0], true);
            flows(d_of[1], false);
        } else {
            if (wave < 4) flows(d_of[0], true);
            else flows(d_of[0], false);
        }
        if (!fine) not_finite = 1;
        {
#pragma unroll
            for (int d = 1; d < kPer; d *= 2) dot_beta += __shfl_xor(dot_beta, d);
            if (threadIdx.x % kPer == 0) dbeta[threadIdx.x / kPer] = dot_beta;
        }
        // the parts that come from and go to other chunks
        if (has_keys) {
            const int d = wave * 16 + at, from = hk * p.Dk + min(d, p.Dk - 1);
            const bool key = d < p.Dk;
            E k_of[4][4], q_of[4][4];
#pragma unroll
            for (int row = 0; row < 4; ++row)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int64_t step = b * p.T + min(chunk * kSteps + row * 16 + group * 4 + r, p.T - 1);
                    k_of[row][r] = static_cast<const E *>(p.k)[step * p.ld_k + from];
                    q_of[row][r] = static_cast<const E *>(p.q)[step * p.ld_q + from];
                }
#pragma unroll
            for (int row = 0; row < 4; ++row) {
                float dot_far[4], dot_later[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = row * 16 + group * 4 + r;
                    const float f = bit_of(alive, i) ? gates.f[i] : 0.0f, t = bit_of(alive, i) ? gates.t[i] : 0.0f;
                    const float k = to_f32(k_of[row][r]), q = to_f32(q_of[row][r]);
                    const float fq = p.scale * f * far_q[row][r], fk = -f * far_k[row][r], e = t * end[row][r];
                    dot_far[r] = f != 0.0f && key ? fmaf(q, fq, k * fk) : 0.0f;
                    dot_later[r] = t != 0.0f && key ? k * e : 0.0f;
                    sum_q[row][r] += f != 0.0f ? fq : 0.0f;
                    sum_k[row][r] += (f != 0.0f ? fk : 0.0f) + (t != 0.0f ? e : 0.0f);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float far = row_sum(dot_far[r]), later = row_sum(dot_later[r]);
                    if (at == 0) {
                        far_of[wave][row * 16 + group * 4 + r] = far;
                        later_of[wave][row * 16 + group * 4 + r] = later;
                    }
                }
            }
        } else {
            far_of[wave][lane] = later_of[wave][lane] = 0.0f;
        }
        const float whole = gates.f[kSteps - 1];
        float through = whole != 0.0f ? whole * dot_states : 0.0f;
        for (int d = 1; d < kWave; d *= 2) through += __shfl_xor(through, d);
        if (lane == 0) extra[wave] = through;
        __syncthreads();
        const bool bad = gates.bad || not_finite;
        auto key_products = [&](const Plane *a, const Frag *keys, Acc (&sum)[4], int which) {
            if (!has_keys) return;
            Frag key[2][PE];
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int n = 0; n < PE; ++n) key[s][n] = FragReader(keys).at(wave, s, n, 2, PE);
#pragma unroll
            for (int row = 0; row < 4; ++row) {
                __builtin_amdgcn_sched_barrier(0);
                if (bad) {
                    unsigned long long pass[4];
                    int hidden = group;                // (the masks are formed here, not kept ready)
                    asm volatile("" : "+v"(hidden));
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int i = row * 16 + hidden * 4 + r;
                        pass[r] = !bit_of(alive, i) ? 0 : (which == 0 ? upto(starts, i) : which == 1 ? from(starts, i) : upto(starts, i) | from(starts, i)) & alive;
                    }
                    sum[row] = careful_rows<PE>(sum[row], a, row, keys, wave, pass);
                } else {
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        if (which == 0 ? s * 32 > row * 16 + 15 : which == 1 ? s * 32 + 31 < row * 16 : false) continue;       // zeros
                        Frag of_a[3];
                        get_frag(a, row, s, of_a);
                        sum[row] = multiply<3, PE>(of_a, key[s], sum[row]);
                    }
                }
            }
        };
        key_products(dN, KT, sum_q, 0);
        key_products(dNT, QT, sum_k, 1);
        if (wave == 0) {
            // (parts of other sequences are 0: f behind the chunk's first start, t before its last)
            const int i = lane, t = chunk * kSteps + i;
            double far = 0.0, later = 0.0, s = 0.0;
#pragma unroll
            for (int w = 0; w < 8; ++w) s += crossing[w][i];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                far += far_of[w][i];
                later += later_of[w][i];
                s += extra[w];
            }
            for (int d = 1; d < kWave; d *= 2) {
                const double behind = __shfl_down(far, d), ahead = __shfl_up(later, d);
                if (i + d < kWave) far += behind;
                if (i >= d) later += ahead;
            }
            later = __shfl_up(later, 1);
            s += far + (i > 0 ? later : 0.0);
            if (t < p.T) {
                const int64_t to = (b * p.T + t) * p.Hv + h;
                p.grad_log_decay[to] = bit_of(alive, i) && !bit_of(starts, i) ? (float)s : 0.0f;
                p.grad_beta[to] = bit_of(alive, i) ? dbeta[i] : 0.0f;
            }
        }
        __syncthreads();
        // X takes the room of dN
        if (kWaves == 4 || wave >= 4) {
            const int row = wave % 4;
#pragma unroll
            for (int tile = 0; tile < 4; ++tile) {
                if (tile > row) continue;
                Four planes[3];
                split(dm[tile], planes);
                const int j = tile * 16 + at;
#pragma unroll
                for (int n = 0; n < 3; ++n) {
                    if (tile < row) *reinterpret_cast<Four *>(&X[n][j][row * 16 + group * 4]) = planes[n];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int i = row * 16 + group * 4 + r;
                        if (tile < row) {
                            X[n][i][j] = planes[n][r];
                        } else if (j <= i) {           // 0 where j = i
                            X[n][i][j] = planes[n][r];
                            X[n][j][i] = planes[n][r];
                        }
                    }
                }
            }
        }
        __syncthreads();
        key_products(X, KT, sum_k, 2);
    }
    // rows of the results through shared memory
    typedef E Row[DK + 8];
    Row *rows = reinterpret_cast<Row *>(lds);
    typedef E Vec __attribute__((ext_vector_type(8)));
    typedef Vec Loose __attribute__((aligned(sizeof(E))));
    auto put = [&](Acc (&sum)[4], void *to, int64_t ld) {
        __syncthreads();
        if (has_keys)
#pragma unroll
            for (int row = 0; row < 4; ++row)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = row * 16 + group * 4 + r;
                    rows[i][wave * 16 + at] = from_f32<E>(bit_of(alive, i) ? sum[row][r] : 0.0f);
                }
        __syncthreads();
        for (int e = threadIdx.x; e < kSteps * (DK / 8); e += kThreads) {
            const int i = e / (DK / 8), d = e % (DK / 8) * 8, t = chunk * kSteps + i;
            if (t >= p.T || d >= p.Dk) continue;
            E *out = const_cast<E *>(row_at<E>(to, ld, b, p.T, t, hk, p.Dk)) + d;
            if (d + 8 <= p.Dk) {
                *reinterpret_cast<Loose *>(out) = *reinterpret_cast<const Vec *>(&rows[i][d]);
            } else {
                for (int c = 0; d + c < p.Dk; ++c) out[c] = rows[i][d + c];
            }
        }
    };
    put(sum_q, p.grad_q, p.ld_gq);
    put(sum_k, p.grad_k, p.ld_gk);
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
    int rc;
    if constexpr (DK == 32) rc = run_back<E, DK, 1>(p, stream);
    else rc = wide_columns<E, DK>(p) ? run_back<E, DK, 2>(p, stream) : run_back<E, DK, 1>(p, stream);
    if (rc || p.chunks == 0) return rc;
    const size_t lds = std::max((6 + kExact<E>) * sizeof(typename Rows<grad_columns(DK)>::Plane), 6 * sizeof(Plane));   // (the results' rows, 64 of DK + 8, are less)
    if (const int failed = make_room_for(reinterpret_cast<const void *>(chunk_grad_kernel<E, DK>), lds)) return failed;
    hipLaunchKernelGGL((chunk_grad_kernel<E, DK>), dim3((unsigned)((int64_t)p.B * p.Hk * p.chunks)), dim3(grad_waves(DK) * kWave), lds, stream, p);
    return launched("delta scan gradient");
}

}  // namespace

int delta_grad_launch(int dtype, const DeltaArgs &p, hipStream_t stream)
{
    return with_dtype(dtype, [&](auto e) { return with_keys(p.Dk, [&](auto dk) { return run<decltype(e), decltype(dk)::value>(p, stream); }); });
}

}  // namespace marl
