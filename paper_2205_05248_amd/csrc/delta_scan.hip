// Gated delta rule, forward: the matrices of every chunk side by side, then the way through the chunks.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "delta.h"

namespace marl {
namespace {

// Gates of a chunk, by one wave, a step a lane.  asked: what they are made of, on its way; put: the gates.
struct GateInputs {
    float log_decay, beta;
    bool live, reset;
    __device__ __forceinline__ GateInputs(const DeltaArgs &p, int64_t b, int h, int chunk)
    {
        const int t = chunk * kSteps + (int)threadIdx.x % kWave;
        const int64_t step = b * p.T + min(t, p.T - 1);
        log_decay = p.log_decay[step * p.Hv + h];
        beta = p.beta[step * p.Hv + h];
        reset = p.reset && p.reset[step];
        live = t < p.T && (!p.filled || p.filled[step]);
    }
    __device__ __forceinline__ void put(ChunkGates &out) const
    {
        const int i = threadIdx.x % kWave;
        float g = live ? log_decay : 0.0f;
        const bool start = live && (reset || g == -__builtin_inff());
        g = start ? 0.0f : g < -200.0f ? -200.0f : g;
        const unsigned long long starts = __ballot(start), so_far = starts << (63 - i);
        const int first = so_far ? i - __clzll((long long)so_far) : 0;             // of the lane's sequence
        double G = g;
        for (int d = 1; d < kWave; d *= 2) {
            const double before = __shfl_up(G, d);
            if (i - d >= first) G += before;
        }
        const int part = __popcll(so_far);
        const double G_end = __shfl(G, 63);
        const int part_end = __shfl(part, 63);
        const float f = part == 0 ? decay_of(G) : 0.0f;
        out.G[i] = G;
        out.f[i] = f;
        out.t[i] = !live ? -1.0f : part == part_end ? decay_of(G_end - G) : 0.0f;
        out.beta[i] = live ? beta : 0.0f;
        const unsigned long long alive = __ballot(live);
        if (i == kSteps - 1) out.whole = f;
        if (i == 0) { out.starts = starts; out.live = alive; out.bad = 0; }
    }
};

// Rows of a chunk as planes in shared memory, zeros in padding and behind Dk.
template <typename E, int DK>
struct KeyRows {
    static constexpr int PE = kExact<E>, LD = DK + 8;
    __bf16 at[PE][kSteps][LD];
    // returns whether all of the lane's entries fit planes
    __device__ __forceinline__ bool fill(const DeltaArgs &p, const void *from, int64_t ld, int64_t b, int hk, int chunk, unsigned long long live)
    {
        typedef E Vec __attribute__((ext_vector_type(8)));
        typedef Vec Loose __attribute__((aligned(sizeof(E))));
        bool fine = true;
        for (int e = threadIdx.x; e < kSteps * (DK / 8); e += kDeltaThreads) {
            const int i = e / (DK / 8), d = e % (DK / 8) * 8;
            float v[8] = {};
            if (bit_of(live, i)) {
                const E *row = row_at<E>(from, ld, b, p.T, chunk * kSteps + i, hk, p.Dk);
                if (d + 8 <= p.Dk) {
                    const Vec x = *reinterpret_cast<const Loose *>(row + d);
#pragma unroll
                    for (int c = 0; c < 8; ++c) v[c] = to_f32(x[c]);
                } else {
#pragma unroll
                    for (int c = 0; c < 8; ++c) v[c] = d + c < p.Dk ? to_f32(row[d + c]) : 0.0f;
                }
            }
#pragma unroll
            for (int c = 0; c < 8; ++c) fine = fine && fits_planes(fabsf(v[c]));
            Frag planes[PE];
            split(v, planes);
#pragma unroll
            for (int n = 0; n < PE; ++n) *reinterpret_cast<Frag *>(&at[n][i][d]) = planes[n];
        }
        return fine;
    }
    __device__ __forceinline__ void row_frag(int tile, int step, Frag (&to)[PE]) const
    {
        const int lane = threadIdx.x % kWave;
#pragma unroll
        for (int n = 0; n < PE; ++n) to[n] = *reinterpret_cast<const Frag *>(&at[n][tile * 16 + lane % 16][step * 32 + lane / 16 * 8]);
    }
    // wave w writes its rows, and every fourth tile of the transposed matrix
    __device__ __forceinline__ void write(Frag *rows, Frag *turned) const
    {
        const int lane = threadIdx.x % kWave, wave = wave_index();
#pragma unroll
        for (int s = 0; s < DK / 32; ++s) {
            Frag f[PE];
            row_frag(wave, s, f);
#pragma unroll
            for (int n = 0; n < PE; ++n) rows[frag_at(wave, s, n, DK / 32, PE)] = f[n];
        }
        if (!turned) return;
        for (int tile = wave; tile < DK / 16; tile += 4)
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int n = 0; n < PE; ++n) {
                    Frag f;
#pragma unroll
                    for (int c = 0; c < 8; ++c) f[c] = at[n][s * 32 + lane / 16 * 8 + c][tile * 16 + lane % 16];
                    turned[frag_at(tile, s, n, 2, PE)] = f;
                }
    }
};

// A 64 x 64 matrix in shared memory as fragments: a wave's rows, or the rows of its transpose; `steps`: which 32 columns hold anything.
template <int PLANES, bool TURNED>
__device__ __forceinline__ void write_square(const float *from, int ld, Frag *to)
{
    const int lane = threadIdx.x % kWave, wave = wave_index(), row = wave * 16 + lane % 16;
    for (int s = 0; s < 2; ++s) {
        if (TURNED ? s * 32 + 31 < wave * 16 : s * 32 > wave * 16 + 15) continue;  // on the other side of the diagonal
        float v[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const int k = s * 32 + lane / 16 * 8 + c;
            v[c] = TURNED ? from[k * ld + row] : from[row * ld + k];
        }
        Frag f[PLANES];
        split(v, f);
#pragma unroll
        for (int n = 0; n < PLANES; ++n) to[frag_at(wave, s, n, 2, PLANES)] = f[n];
    }
}

// A workgroup per key head and chunk: K and Q as fragments, and N and P of every value head that shares them, four at a time.  Bound by what it
// writes, 37 or 74 KB for the squares of a head and three or four matrices of its keys: 0.87 GB of 4 x 8192 x 16 heads x 128 x 128 bf16 with what the backward
// pass needs in 215 us, 4.0 TB/s (with a plane of P less 207 us, 253 with two workgroups a compute unit, which is what shared memory had room for before
// N and A took that of K and Q, 222 with three; with 128 registers some 25 are spilled, which costs fp32 rows, three planes each, more than the fourth
// workgroup gives).
template <typename E, int DK>
__global__ __launch_bounds__(kDeltaThreads, kExact<E> == 1 ? 4 : 3) void chunk_kernel(DeltaArgs p)
{
    constexpr int PE = kExact<E>, LN = kSteps + 1, kOrder = PE == 1 ? 0 : 2;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    auto &K = *reinterpret_cast<KeyRows<E, DK> *>(lds);
    auto &Q = *reinterpret_cast<KeyRows<E, DK> *>(lds + sizeof(K));
    float *A = reinterpret_cast<float *>(lds), *N = A + kSteps * LN;
    __shared__ ChunkGates gates_of[4];
    __shared__ int bad_rows, bad;
    const int chunk = (int)(blockIdx.x % p.chunks), hk = (int)(blockIdx.x / p.chunks % p.Hk);
    const int64_t b = blockIdx.x / p.chunks / p.Hk;
    const int lane = threadIdx.x % kWave, wave = wave_index(), at = lane % 16, group = lane / 16;
    const int shared = p.Hv / p.Hk;
    if (threadIdx.x == 0) bad_rows = 0;
    unsigned long long live;
    {
        const GateInputs inputs(p, b, hk * shared + min(wave, shared - 1), chunk);
        live = __ballot(inputs.live);
        __syncthreads();
        bool fine = K.fill(p, p.k, p.ld_k, b, hk, chunk, live);
        fine = Q.fill(p, p.q, p.ld_q, b, hk, chunk, live) && fine;
        if (!fine) bad_rows = 1;
        inputs.put(gates_of[wave]);
    }
    __syncthreads();
    Acc kk[4] = {}, qk[4] = {};
#pragma unroll
    for (int s = 0; s < DK / 32; ++s) {
        Frag k[PE], q[PE];
        K.row_frag(wave, s, k);
        Q.row_frag(wave, s, q);
#pragma unroll
        for (int tile = 0; tile < 4; ++tile) {
            if (tile > wave) continue;
            Frag other[PE];
            K.row_frag(tile, s, other);
            kk[tile] = multiply<PE, PE, kOrder>(k, other, kk[tile]);
            qk[tile] = multiply<PE, PE, kOrder>(q, other, qk[tile]);
        }
    }
    K.write(p.K + (int64_t)blockIdx.x * key_frags(DK, PE), p.KT + (int64_t)blockIdx.x * key_frags(DK, PE));
    Q.write(p.Q + (int64_t)blockIdx.x * key_frags(DK, PE), p.QT ? p.QT + (int64_t)blockIdx.x * key_frags(DK, PE) : nullptr);
    __syncthreads();                                   // A and N take the room of K and Q
    for (int member = 0; member < shared; ++member) {
        const int64_t record = (b * p.Hv + hk * shared + member) * p.chunks + chunk;
        if (member > 0) {
            if (member % 4 == 0) {
                __syncthreads();
                GateInputs(p, b, hk * shared + min(member + wave, shared - 1), chunk).put(gates_of[wave]);
            }
            __syncthreads();
        }
        ChunkGates &gates = gates_of[member % 4];
        if (threadIdx.x == 0) bad = bad_rows;
        const unsigned long long starts = gates.starts;
        unsigned long long before[4];                  // steps that hand something to the lane's rows
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = wave * 16 + group * 4 + r;
            before[r] = bit_of(live, i) ? upto(starts, i) & live : 0;
        }
        // P through the room of N, then A
        bool fine = true;
#pragma unroll
        for (int tile = 0; tile < 4; ++tile) {
            const int j = tile * 16 + at;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = wave * 16 + group * 4 + r;
                float a = 0.0f, v = 0.0f;
                if (tile <= wave) {
                    const bool on = bit_of(before[r], j);
                    const float e = decay_of(gates.G[i] - gates.G[j]);
                    a = on && j < i ? e * kk[tile][r] : 0.0f;
                    v = on ? p.scale * e * qk[tile][r] : 0.0f;
                    fine = fine && fits_planes(max_of(fabsf(a), fabsf(v)));
                }
                A[i * LN + j] = a;
                N[i * LN + j] = v;
            }
        }
        __syncthreads();
        write_square<3, false>(N, LN, p.P + record * square_frags(3));
        if (p.PT) write_square<3, true>(N, LN, p.PT + record * square_frags(3));
        // blocks on the diagonal: N_i = A_i - sum_j A_ij beta_j N_j, a column a lane
        float n[16];
        {
            const float *own = A + (wave * 16) * LN + wave * 16;
            float column[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) column[i] = own[i * LN + at];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float v = column[i];
#pragma unroll
                for (int j = 0; j < i; ++j) v = fmaf(-own[i * LN + j], n[j], v);
                v = i > at ? v : 0.0f;
                fine = fine && fits_planes(fabsf(v));
                n[i] = v * gates.beta[wave * 16 + i];
                column[i] = v;
            }
            __syncthreads();                           // P has been read
            if (group == 0)
#pragma unroll
                for (int i = 0; i < 16; ++i) N[(wave * 16 + i) * LN + wave * 16 + at] = column[i];
            for (int e = lane; e < 16 * kSteps; e += kWave)                        // above the diagonal
                if (e % kSteps >= wave * 16 + 16) N[(wave * 16 + e / kSteps) * LN + e % kSteps] = 0.0f;
        }
        __syncthreads();
        // block columns: N_ij = (I - N_ii beta) (A_ij - sum_m A_im beta_m N_mj), downwards
        for (int i = wave + 1; i < 4; ++i) {
            Acc c;
#pragma unroll
            for (int r = 0; r < 4; ++r) c[r] = A[(i * 16 + group * 4 + r) * LN + wave * 16 + at];
            for (int m = wave; m < i; ++m)
                c = product(c, [&](int row, int k) { return -A[(i * 16 + row) * LN + m * 16 + k] * gates.beta[m * 16 + k]; },
                            [&](int k, int col) { return N[(m * 16 + k) * LN + wave * 16 + col]; });
#pragma unroll
            for (int r = 0; r < 4; ++r) N[(i * 16 + group * 4 + r) * LN + wave * 16 + at] = c[r];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            c = product(c, [&](int row, int k) { return -N[(i * 16 + row) * LN + i * 16 + k] * gates.beta[i * 16 + k]; },
                        [&](int k, int col) { return N[(i * 16 + k) * LN + wave * 16 + col]; });
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int r = 0; r < 4; ++r) N[(i * 16 + group * 4 + r) * LN + wave * 16 + at] = c[r];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            fine = fine && all_finite(c);
        }
        if (!fine) bad = 1;
        __syncthreads();
        if (bad && wave == 0) {                        // again without anything that is not one of the sequence's steps in between
            for (int i = 0; i < kSteps; ++i) {
                float v = 0.0f;
                if (lane < i && joined(starts, i, lane)) {
                    v = A[i * LN + lane];
                    for (int j = lane + 1; j < i; ++j)
                        if (bit_of(live, j)) v = fmaf(-A[i * LN + j] * gates.beta[j], N[j * LN + lane], v);
                }
                N[i * LN + lane] = v;
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
        }
        if (threadIdx.x == 0) gates.bad = bad;
        __syncthreads();
        write_square<3, false>(N, LN, p.N + record * square_frags(3));
        if (p.NT) write_square<3, true>(N, LN, p.NT + record * square_frags(3));
        const int *from = reinterpret_cast<const int *>(&gates);
        int *to = reinterpret_cast<int *>(p.gates + record);
        for (int e = threadIdx.x; e < (int)(sizeof(ChunkGates) / 4); e += kDeltaThreads) to[e] = from[e];
    }
}

// The chunks of one head one after the other, for 16 NT value columns: tile n of a lane's column l % 16 is column NT (l % 16) + n.  Wave w has
// rows 16 w on of the chunk, and rows w DK / 4 on of the state, which stays in its accumulators; the others read it as planes from shared memory.
// What a phase needs from memory is asked for where the same phase of the chunk before has used its registers, a whole chunk ahead, and
// whether there is another chunk or not: behind a branch the compiler would wait for it at the next wait of any kind.
// Bound by the chain of a chunk: three barriers, between them products that wait for the splitting of what the other waves made; at 128 keys and columns a
// chunk takes 2.5 us with 16 columns (20011 steps, 16 heads, bf16: 775 us, 128 workgroups on 256 compute units; 360 vector and 54 matrix instructions a
// wave) and 5.4 with 32 (4 x 8192, with keep: 697 us, 900 and 108 instructions, waves wait 33 % of their cycles, the matrix pipe is busy for 13 %).  Everything
// at hand a chunk ahead takes 1.4 times the registers that a third workgroup on a compute unit would leave: with 168 they spill, 88 -> 196 us of the 320 x 120
// batch with 4 heads of 16.  fp16 with 128 keys spills with 256 too, and has a compute unit for a workgroup: 450 -> 293 us of 4096 steps, 16 heads with keep.
template <typename E, int DK, int NT, bool KEEP>
__global__ __launch_bounds__(kDeltaThreads, (NT == 1 ? kExact<E> * DK <= 192 : DK == 32) ? 2 : 1) void scan_kernel(DeltaArgs p)
{
    constexpr int PE = kExact<E>, KS = DK / 32, LS = DK + 8, LU = kSteps + 8, C = 16 * NT;
    constexpr int kTiles = (DK + 63) / 64;             // of the state, for a wave; of DK = 32 two waves have one
    extern __shared__ __attribute__((aligned(16))) char lds[];
    typedef __bf16 StatePlane[C][LS];
    typedef __bf16 StepPlane[C][LU];
    StatePlane *S = reinterpret_cast<StatePlane *>(lds);                           // [3], columns of the state
    StepPlane *R = reinterpret_cast<StepPlane *>(lds + 3 * sizeof(StatePlane)), *U = R + 3, *Ue = U + 3;       // [3] each
    __shared__ int not_finite[2];
    const int lane = threadIdx.x % kWave, wave = wave_index(), at = lane % 16, group = lane / 16, zero = hidden_zero();
    const Place place = place_of((int64_t)p.B * p.Hv, p.Dv, C);
    if (place.head < 0) return;                        // the whole workgroup
    const int64_t head = place.head, b = head / p.Hv;
    const int col = place.first + at * NT, h = (int)(head % p.Hv), hk = h / (p.Hv / p.Hk), DV = padded_values(p.Dv);
    const int64_t key_head = b * p.Hk + hk;
    const bool has_state = DK >= 64 || wave * 16 < DK;
    Acc state[kTiles][NT] = {};
    if (p.s_first && has_state)
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = (wave * kTiles + tile) * 16 + group * 4 + r;
                float v[NT] = {};
                if (d < p.Dk) read_columns<float, NT>(p.s_first + (head * p.Dk + d) * p.Dv, col, p.Dv, v);
#pragma unroll
                for (int n = 0; n < NT; ++n) state[tile][n][r] = v[n];
            }
    Frag k[KS][PE], q[KS][PE], n_of[2][3], p_of[2][3], kt[kTiles][2][PE];
    Columns<E, NT> v[4];
    Acc f_next, t_next, beta_next;
    float whole_next;
    int bad_next;
    const unsigned of_row = (wave * 16 + group * 4) * 4u, row_bytes = (unsigned)p.ld_v * (unsigned)sizeof(E);
    const unsigned first_v = (wave * 16 + group * 4) * row_bytes + (unsigned)min(col, p.Dv - NT) * (unsigned)sizeof(E);
    auto load_start = [&](int chunk) {
        const ChunkGates *g = p.gates + head * p.chunks + chunk;
        const FragReader K(p.K + (key_head * p.chunks + chunk) * key_frags(DK, PE)), Q(p.Q + (key_head * p.chunks + chunk) * key_frags(DK, PE));
        f_next = read_at<Acc>(g->f, of_row);
        t_next = read_at<Acc>(g->t, of_row);
        beta_next = read_at<Acc>(g->beta, of_row);
        whole_next = read_at<float>(&g->whole, (unsigned)zero);
        bad_next = read_at<int>(&g->bad, (unsigned)zero);
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int n = 0; n < PE; ++n) {
                k[s][n] = K.at(wave, s, n, KS, PE);
                q[s][n] = Q.at(wave, s, n, KS, PE);
            }
        const E *rows = row_at<E>(p.v, p.ld_v, b, p.T, chunk * kSteps, h, p.Dv);
        const int last = p.T - chunk * kSteps;         // rows behind it are not read: the first one is instead
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r].load(rows, wave * 16 + group * 4 + r < last ? first_v + r * row_bytes : first_v - (wave * 16 + group * 4) * row_bytes);
    };
    auto load_n = [&](int chunk) {                     // (what lies on the other side of the diagonal is never written, and not used)
        const FragReader N(p.N + (head * p.chunks + chunk) * square_frags(3));
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int n = 0; n < 3; ++n) n_of[s][n] = N.at(wave, s, n, 2, 3);
    };
    auto load_end = [&](int chunk) {
        const FragReader P(p.P + (head * p.chunks + chunk) * square_frags(3)), KT(p.KT + (key_head * p.chunks + chunk) * key_frags(DK, PE));
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int n = 0; n < PE; ++n) kt[tile][s][n] = KT.at((wave * kTiles + tile) % (DK / 16), s, n, 2, PE);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int n = 0; n < 3; ++n) p_of[s][n] = P.at(wave, s, n, 2, 3);
    };
    auto share_state = [&] {
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                Four planes[3];
                split(state[tile][n], planes);
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
    if (p.chunks > 0) {
        load_start(0);
        load_n(0);
        load_end(0);
    }
    if (has_state) share_state();
    if (threadIdx.x < 2) not_finite[threadIdx.x] = 0;
    __syncthreads();
    for (int chunk = 0; chunk < p.chunks; ++chunk) {
        const int64_t record = head * p.chunks + chunk;
        const int next = min(chunk + 1, p.chunks - 1);
        const Acc f = f_next, t = t_next, beta = beta_next;
        const float whole = whole_next;
        const bool bad = __builtin_amdgcn_readfirstlane(bad_next) != 0;
        // R = V - f K S
        Sums<2> ks[NT], qs[NT];
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                Frag of_state[3];
#pragma unroll
                for (int m = 0; m < 3; ++m) of_state[m] = *reinterpret_cast<const Frag *>(&S[m][n * 16 + at][s * 32 + group * 8]);
                multiply_into(ks[n], k[s], of_state);
                multiply_into(qs[n], q[s], of_state);
            }
        Acc m[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const Acc of_k = total(ks[n]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float value = v[r].at(n, col, p.Dv);
                m[n][r] = t[r] < 0.0f ? 0.0f : f[r] == 0.0f ? value : fmaf(-f[r], of_k[r], value);
            }
            const Acc minus = -(beta * m[n]);
            Four planes[3];
            split(minus, planes);
            share_steps(R, planes, n);
            if (!all_finite(minus)) not_finite[0] = 1;
        }
        load_start(next);
        if (KEEP && has_state) {
            float *to = p.S + record * DK * DV;
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float c[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) c[n] = state[tile][n][r];
                    write_columns<float, NT>(to, ((wave * kTiles + tile) * 16 + group * 4 + r) * DV + col, DK * DV, c);
                }
        }
        __syncthreads();
        // M = R - N (beta R), U = beta M
        Frag of_r[2][NT][3];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n) steps_frag(R, n, s, of_r[s][n]);
        if (bad || not_finite[0]) {
            const unsigned long long starts = p.gates[record].starts, live = p.gates[record].live;
            unsigned long long pass[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = wave * 16 + group * 4 + r;
                pass[r] = bit_of(live, i) ? upto(starts, i) & live & ~(1ull << i) : 0;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) m[n] = careful_multiply<3, 3>(m[n], p.N + record * square_frags(3), wave, R[0][n * 16 + at], C * LU, pass);
        } else {
            Sums<2> nr[NT];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (s * 32 > wave * 16) continue;
#pragma unroll
                for (int n = 0; n < NT; ++n) multiply_into(nr[n], n_of[s], of_r[s][n]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) m[n] += total(nr[n]);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const Acc u = beta * m[n];
            Acc to_end;
#pragma unroll
            for (int r = 0; r < 4; ++r) to_end[r] = t[r] > 0.0f || t[r] != t[r] ? t[r] * u[r] : 0.0f;
            Four planes[3], end_planes[3];
            split(u, planes);
            split(to_end, end_planes);
            share_steps(U, planes, n);
            share_steps(Ue, end_planes, n);
            if (!all_finite(u)) not_finite[1] = 1;
        }
        load_n(next);
        if (KEEP) {
            float *to = p.M + record * kSteps * DV;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float c[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) c[n] = m[n][r];
                write_columns<float, NT>(to, (wave * 16 + group * 4 + r) * DV + col, kSteps * DV, c);
            }
        }
        __syncthreads();
        // O = scale f Q S + P U,  S <- f_63 S + K' (t U)
        Frag of_e[2][NT][3], of_u[2][NT][3];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n) steps_frag(Ue, n, s, of_e[s][n]);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n) steps_frag(U, n, s, of_u[s][n]);
        Acc o[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const Acc of_q = total(qs[n]);
#pragma unroll
            for (int r = 0; r < 4; ++r) o[n][r] = f[r] == 0.0f ? 0.0f : p.scale * f[r] * of_q[r];
        }
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) state[tile][n][r] = whole == 0.0f ? 0.0f : whole * state[tile][n][r];
        if (bad || not_finite[1]) {
            const unsigned long long starts = p.gates[record].starts, live = p.gates[record].live;
            unsigned long long pass[4];
            if (has_state) {
#pragma unroll
                for (int r = 0; r < 4; ++r) pass[r] = upto(starts, kSteps - 1) & live;
#pragma unroll
                for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        state[tile][n] = careful_multiply<PE, 3>(state[tile][n], p.KT + (key_head * p.chunks + chunk) * key_frags(DK, PE),
                                                                 wave * kTiles + tile, Ue[0][n * 16 + at], C * LU, pass);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = wave * 16 + group * 4 + r;
                pass[r] = bit_of(live, i) ? upto(starts, i) & live : 0;
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) o[n] = careful_multiply<3, 3>(o[n], p.P + record * square_frags(3), wave, U[0][n * 16 + at], C * LU, pass);
        } else {
            if (has_state) {
                Sums<2> ku[kTiles][NT];
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int tile = 0; tile < kTiles; ++tile) multiply_into(ku[tile][n], kt[tile][s], of_e[s][n]);
#pragma unroll
                for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
                    for (int n = 0; n < NT; ++n) state[tile][n] += total(ku[tile][n]);
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (s * 32 > wave * 16) continue;
#pragma unroll
                for (int n = 0; n < NT; ++n) o[n] = multiply<3, 3>(p_of[s], of_u[s][n], o[n]);
            }
        }
        load_end(next);
        if (has_state) share_state();
        const RowsOut<E, NT> out(p, p.o, p.ld_o, b, chunk, h);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float c[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) c[n] = t[r] < 0.0f ? 0.0f : o[n][r];
            out.put(wave * 16 + group * 4 + r, col, c);
        }
        if (threadIdx.x == 0) not_finite[0] = 0;       // read before the barrier above, written after the one below
        __syncthreads();
        if (threadIdx.x == 0) not_finite[1] = 0;
    }
    if (p.s_last && has_state)
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = (wave * kTiles + tile) * 16 + group * 4 + r;
                float v[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) v[n] = state[tile][n][r];
                if (d < p.Dk) write_columns<float, NT>(p.s_last + (head * p.Dk + d) * p.Dv, col, p.Dv, v);
            }
}

template <typename E, int DK, int NT>
int run_scan(const DeltaArgs &p, hipStream_t stream)
{
    const size_t lds = (size_t)16 * NT * (3 * (DK + 8) + 9 * (kSteps + 8)) * sizeof(__bf16);
    const auto go = [&](auto kernel) {
        if (const int rc = make_room_for(reinterpret_cast<const void *>(kernel), lds)) return rc;
        hipLaunchKernelGGL(kernel, dim3(places((int64_t)p.B * p.Hv, p.Dv, 16 * NT)), dim3(kDeltaThreads), lds, stream, p);
        return launched("delta scan");
    };
    return p.S ? go(scan_kernel<E, DK, NT, true>) : go(scan_kernel<E, DK, NT, false>);
}

template <typename E, int DK>
int run(const DeltaArgs &p, hipStream_t stream)
{
    if (p.chunks > 0) {
        const size_t lds = std::max(2 * sizeof(KeyRows<E, DK>), (size_t)2 * kSteps * (kSteps + 1) * sizeof(float));
        if (const int rc = make_room_for(reinterpret_cast<const void *>(chunk_kernel<E, DK>), lds)) return rc;
        hipLaunchKernelGGL((chunk_kernel<E, DK>), dim3((unsigned)((int64_t)p.B * p.Hk * p.chunks)), dim3(kDeltaThreads), lds, stream, p);
    }
    return wide_columns<E, DK>(p) ? run_scan<E, DK, 2>(p, stream) : run_scan<E, DK, 1>(p, stream);
}

}  // namespace

int delta_scan_launch(int dtype, const DeltaArgs &p, hipStream_t stream)
{
    return with_dtype(dtype, [&](auto e) { return with_keys(p.Dk, [&](auto dk) { return run<decltype(e), decltype(dk)::value>(p, stream); }); });
}

}  // namespace marl
