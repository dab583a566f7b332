// Gated linear recurrence: h[t] = a[t] h[t-1] + beta[t] sigmoid(i[t]) x[t], its backward pass and its form for one step.
#include <hip/hip_runtime.h>

#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "device_math.h"
#include "operator_types.h"

namespace marl {
namespace {

// The shape of the work.  A workgroup (a "unit") takes CT = 8 V channels, V of them 16 bytes of a row, over a span of
// steps: eight lanes share a row, so a load instruction brings 128 bytes of each of eight rows, and a lane walks Tc steps
// that follow one another.  Groups of eight lanes, then waves, then units follow one another in time.  What a
// stretch of steps does to the state is h -> A h + H, and stretches compose; so a lane composes its own steps, eight groups
// compose by lane exchange, the waves through shared memory, and units through memory (see look_back).  The inputs are read
// once and stay in registers until the state at the unit's start is known.
// Narrow and long units: the number of units of one sequence in flight, which is what look_back walks over, is small.
template <typename E>
struct Span {
    static constexpr int V = 16 / (int)sizeof(E);
    static constexpr int CT = 8 * V;
};

constexpr int kElements = 32, kElementsBack = 16;      // of a lane: V channels x Tc steps (the backward pass keeps more of each)
constexpr int kMostWaves = 8;

template <typename E> constexpr int steps_of_lane(bool back) { return (back ? kElementsBack : kElements) / Span<E>::V; }

// Waves of a unit: enough for T, at most kMostWaves.
inline int waves_for(int T, int lane_steps)
{
    int w = 1;
    while (w < kMostWaves && w * 8 * lane_steps < T) w *= 2;
    return w;
}

typedef unsigned long long Word;       // A with its sign bit set, above H: one 64-bit store says both.  0: not there yet

struct ScanArgs {
    int B, T, C;
    int tiles, sequences, units;       // channel tiles, B tiles, units of a sequence
    const void *x, *r, *i;
    int64_t ld_x, ld_r, ld_i;
    const float *lam;
    float decay;
    const uint8_t *reset, *filled;
    const float *h_first;
    void *y;
    int64_t ld_y;
    float *h_last;
    float *states;                     // [B, kept, C] state before each `keep`-th step
    int keep, kept;
    unsigned *ticket;                  // order in which units begin
    Word *words;                       // [units, sequences, CT]
    // backward pass
    const void *grad_y;
    int64_t ld_gy;
    const float *grad_h_last;
    void *grad_x, *grad_r, *grad_i;
    int64_t ld_gx, ld_gr, ld_gi;
    float *lam_part;                   // [B units, C]
    float *grad_lam, *grad_h_first;
};

__device__ __forceinline__ float rate_of(float lam, float decay)
{
    return decay * (lam > 20.0f ? lam : log1pf(expf(lam)));      // (above 20 the difference is below half a step)
}

// sigmoid(v) and its complement, each to fp32 accuracy at both ends.
struct Sigmoid { float s, c; };
__device__ __forceinline__ Sigmoid sigmoid2(float v)
{
    const float e = fminf(__builtin_amdgcn_exp2f(-kLog2e * v), 1e37f);
    const float s = __builtin_amdgcn_rcpf(1.0f + e);
    return {s, e * s};
}

// 1 - exp(y) for y <= 0.  Near 0 the difference would cancel: there the series, whose next term is below 2^-25.
__device__ __forceinline__ float one_minus_exp(float y, float exp_y)
{
    float p = fmaf(y, 1.0f / 7.0f, 1.0f);
    p = fmaf(y * (1.0f / 6.0f), p, 1.0f);
    p = fmaf(y * 0.2f, p, 1.0f);
    p = fmaf(y * 0.25f, p, 1.0f);
    p = fmaf(y * (1.0f / 3.0f), p, 1.0f);
    p = fmaf(y * 0.5f, p, 1.0f);
    return y > -0.35f ? -y * p : 1.0f - exp_y;
}

struct Gates { Sigmoid sr, si; float a, inv_beta, beta; };
__device__ __forceinline__ Gates gates_of(float r, float i, float rate)
{
    Gates g;
    g.sr = sigmoid2(r);
    g.si = sigmoid2(i);
    const float L = -rate * g.sr.s;
    g.a = __builtin_amdgcn_exp2f(kLog2e * L);
    const float om = one_minus_exp(2.0f * L, g.a * g.a);
    g.inv_beta = __builtin_amdgcn_rsqf(fmaxf(om, 1e-30f));     // a gate that is shut has om = 0: beta 0, and no infinity
    g.beta = om * g.inv_beta;
    return g;
}

// 16 bytes of a row; entries beyond the last channel are zero and not stored.
template <typename E, bool VEC>
struct Row {
    static constexpr int V = Span<E>::V;
    typedef E Vec __attribute__((ext_vector_type(V)));
    Vec v;
    __device__ __forceinline__ void load(const void *base, int64_t at, int left)
    {
        const E *p = static_cast<const E *>(base) + at;
        if constexpr (VEC) {
            v = *reinterpret_cast<const Vec *>(p);
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = k < left ? p[k] : (E)0.0f;
        }
    }
    __device__ __forceinline__ void store(void *base, int64_t at, int left) const
    {
        E *p = static_cast<E *>(base) + at;
        if constexpr (VEC) {
            *reinterpret_cast<Vec *>(p) = v;
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k < left) p[k] = v[k];
        }
    }
};

__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// What a step does to the state.  kPast: behind the last step; as padding, but nothing is stored.
enum Kind { kPast, kPadding, kStart, kOrdinary };
__device__ __forceinline__ Kind kind_of(const ScanArgs &p, int64_t b, int t)
{
    if (t >= p.T) return kPast;
    const int64_t row = b * p.T + t;
    if (p.filled && !p.filled[row]) return kPadding;
    return p.reset && p.reset[row] ? kStart : kOrdinary;
}

__device__ __forceinline__ Word word_of(float A, float H)
{
    return (Word)(__float_as_uint(A) | 0x80000000u) << 32 | __float_as_uint(H);
}
__device__ __forceinline__ void publish(Word *at, float A, float H) { __hip_atomic_store(at, word_of(A, H), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ Word peek(const Word *at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The state at the start of a unit, a lane per channel.  Units publish (A, H) of their own steps at once, without waiting
// for anything, and (0, h) of the state behind them when they know it; A = 0 says that nothing before matters.  Walking
// backwards from unit `before` over whichever is there, `stride` words apart, until A = 0; the first unit publishes (0, h) alone.  A unit
// waits only for units whose tickets are lower, and they began before it: each wait ends.
__device__ __forceinline__ float look_back(const Word *words, int before, int64_t stride, bool mine)
{
    constexpr int kAtOnce = 8;
    float A = 1.0f, H = 0.0f;
    bool open = mine;
    for (int k = before; k >= 0 && __any(open); k -= kAtOnce) {
        Word w[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) w[j] = open && k - j >= 0 ? peek(words + (int64_t)(k - j) * stride) : 0;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (k - j < 0) break;
            while (__any(open && w[j] == 0)) {
                __builtin_amdgcn_s_sleep(1);
                if (open && w[j] == 0) w[j] = peek(words + (int64_t)(k - j) * stride);
            }
            if (open) {
                const float a = __uint_as_float((unsigned)(w[j] >> 32) & 0x7fffffffu);
                H = fmaf(A, __uint_as_float((unsigned)w[j]), H);
                A *= a;
                open = a != 0.0f;
            }
        }
    }
    return H;
}

// Clears the words and the ticket and puts the first states aside (h_last may be h_first, and the last unit may be done with it
// before the first one has begun).
__global__ __launch_bounds__(256) void scan_begin_kernel(Word *words, int64_t n_words, unsigned *ticket, const float *h_first, float *aside, int64_t n_states)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id == 0) *ticket = 0;
    if (id < n_words) words[id] = 0;
    if (id < n_states) aside[id] = h_first ? h_first[id] : 0.0f;
}

// Unit of a workgroup: sequences advance side by side, time outermost.
struct Place { int seq, unit, b, c0; };
template <typename E, bool CHAIN>
__device__ __forceinline__ Place place_of(const ScanArgs &p, int *shared)
{
    int id = blockIdx.x;
    if constexpr (CHAIN) {
        if (threadIdx.x == 0) *shared = (int)atomicAdd(p.ticket, 1u);
        lds_barrier();
        id = *shared;
    }
    const int seq = id % p.sequences;
    return {seq, id / p.sequences, seq / p.tiles, seq % p.tiles * Span<E>::CT};
}

template <typename E, bool VEC, int NW, bool CHAIN>
__global__ __launch_bounds__(NW * kWave, 4) void scan_kernel(ScanArgs p)
{
    constexpr int V = Span<E>::V, CT = Span<E>::CT, Tc = steps_of_lane<E>(false);
    __shared__ float rate_s[CT], A_s[NW][CT], H_s[NW][CT], carry_s[NW][CT];
    __shared__ int id_s;
    const Place at = place_of<E, CHAIN>(p, &id_s);
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, group = lane / 8, cl = lane % 8 * V;
    const int c = at.c0 + cl, left = p.C - c, first = at.unit * (NW * 8 * Tc), t0 = first + (wave * 8 + group) * Tc;
    Row<E, VEC> x[Tc], r[Tc], i[Tc];
    Kind kind[Tc];
#pragma unroll
    for (int j = 0; j < Tc; ++j) {
        kind[j] = left > 0 ? kind_of(p, at.b, t0 + j) : kPast;
        if (kind[j] > kPadding) {
            const int64_t row = (int64_t)at.b * p.T + t0 + j;
            x[j].load(p.x, row * p.ld_x + c, left);
            r[j].load(p.r, row * p.ld_r + c, left);
            i[j].load(p.i, row * p.ld_i + c, left);
        }
    }
    for (int k = threadIdx.x; k < CT; k += NW * kWave) rate_s[k] = at.c0 + k < p.C ? rate_of(p.lam[at.c0 + k], p.decay) : 0.0f;
    lds_barrier();
    float a[Tc][V], u[Tc][V], A[V], H[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { A[v] = 1.0f; H[v] = 0.0f; }
#pragma unroll
    for (int j = 0; j < Tc; ++j) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            a[j][v] = 1.0f;
            u[j][v] = 0.0f;
        }
        if (kind[j] > kPadding) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Gates g = gates_of(to_f32(r[j].v[v]), to_f32(i[j].v[v]), rate_s[cl + v]);
                const float in = g.si.s * to_f32(x[j].v[v]);
                a[j][v] = kind[j] == kStart ? 0.0f : g.a;
                u[j][v] = kind[j] == kStart ? in : g.beta * in;
                H[v] = fmaf(a[j][v], H[v], u[j][v]);
                A[v] *= a[j][v];
            }
        }
    }
    // what the groups before this one do: composed over the groups of the wave, then shifted by one
    float A_before[V], H_before[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int d = 8; d < kWave; d *= 2) {
            const float pA = __shfl_up(A[v], d), pH = __shfl_up(H[v], d);
            if (lane >= d) {
                H[v] = fmaf(A[v], pH, H[v]);
                A[v] *= pA;
            }
        }
        A_before[v] = __shfl_up(A[v], 8);
        H_before[v] = __shfl_up(H[v], 8);
        if (lane < 8) { A_before[v] = 1.0f; H_before[v] = 0.0f; }
        if (lane >= kWave - 8) { A_s[wave][cl + v] = A[v]; H_s[wave][cl + v] = H[v]; }
    }
    lds_barrier();
    if (wave == 0) {
        const int ch = at.c0 + lane;
        const bool mine = lane < CT && ch < p.C;
        float Aw = 1.0f, Hw = 0.0f;
        if (mine)
            for (int w = 0; w < NW; ++w) { Hw = fmaf(A_s[w][lane], Hw, H_s[w][lane]); Aw *= A_s[w][lane]; }
        float h = 0.0f;
        if constexpr (CHAIN) {
            const int64_t stride = (int64_t)p.sequences * CT;
            Word *own = p.words + (int64_t)at.seq * CT + lane;
            if (at.unit > 0) {
                if (mine) publish(own + at.unit * stride, Aw, Hw);
                h = look_back(own, at.unit - 1, stride, mine);
            } else if (mine) {
                h = p.h_first[(int64_t)at.b * p.C + ch];
            }
            if (mine) publish(own + at.unit * stride, 0.0f, fmaf(Aw, h, Hw));
        } else if (mine && p.h_first) {
            h = p.h_first[(int64_t)at.b * p.C + ch];
        }
        if (mine) {
            for (int w = 0; w < NW; ++w) {
                carry_s[w][lane] = h;
                const int t = first + w * 8 * Tc;
                if (t < p.T && t % p.keep == 0) p.states[((int64_t)at.b * p.kept + t / p.keep) * p.C + ch] = h;
                h = fmaf(A_s[w][lane], h, H_s[w][lane]);
            }
            if (p.h_last && at.unit == p.units - 1) p.h_last[(int64_t)at.b * p.C + ch] = h;
        }
    }
    lds_barrier();
    if (left <= 0) return;
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = fmaf(A_before[v], carry_s[wave][cl + v], H_before[v]);
#pragma unroll
    for (int j = 0; j < Tc; ++j) {
        if (kind[j] == kPast) continue;
        Row<E, VEC> y;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            h[v] = fmaf(a[j][v], h[v], u[j][v]);
            y.v[v] = from_f32<E>(kind[j] == kPadding ? 0.0f : h[v]);
        }
        y.store(p.y, ((int64_t)at.b * p.T + t0 + j) * p.ld_y + c, left);
    }
}

// Backward pass.  D[t] = a[t] dL/dh[t] is what reaches h[t-1]: D[t] = a[t] (grad_y[t] + D[t+1]), the same kind of chain
// backwards in time.  h is formed again inside the unit from the state kept at its start.
template <typename E, bool VEC, int NW, bool CHAIN>
__global__ __launch_bounds__(NW * kWave) void scan_grad_kernel(ScanArgs p)
{
    constexpr int V = Span<E>::V, CT = Span<E>::CT, Tc = steps_of_lane<E>(true);
    __shared__ float rate_s[CT], A_s[NW][CT], H_s[NW][CT], R_s[NW][CT], carry_s[NW][CT], after_s[NW][CT];
    __shared__ int id_s;
    const Place at = place_of<E, CHAIN>(p, &id_s);
    const int unit = p.units - 1 - at.unit;                    // the last steps first
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, group = lane / 8, cl = lane % 8 * V;
    const int c = at.c0 + cl, left = p.C - c, t0 = unit * (NW * 8 * Tc) + (wave * 8 + group) * Tc;
    Row<E, VEC> x[Tc], r[Tc], i[Tc], g[Tc];
    Kind kind[Tc];
#pragma unroll
    for (int j = 0; j < Tc; ++j) {
        kind[j] = left > 0 ? kind_of(p, at.b, t0 + j) : kPast;
        if (kind[j] > kPadding) {
            const int64_t row = (int64_t)at.b * p.T + t0 + j;
            r[j].load(p.r, row * p.ld_r + c, left);
            i[j].load(p.i, row * p.ld_i + c, left);
            x[j].load(p.x, row * p.ld_x + c, left);
            g[j].load(p.grad_y, row * p.ld_gy + c, left);
        }
    }
    for (int k = threadIdx.x; k < CT; k += NW * kWave) rate_s[k] = at.c0 + k < p.C ? rate_of(p.lam[at.c0 + k], p.decay) : 0.0f;
    lds_barrier();
    Gates gate[Tc][V];
    float u[Tc][V], A[V], H[V], R[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { A[v] = 1.0f; H[v] = 0.0f; R[v] = 0.0f; }
#pragma unroll
    for (int j = 0; j < Tc; ++j) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            gate[j][v].a = 1.0f;
            u[j][v] = 0.0f;
        }
        if (kind[j] > kPadding) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                Gates &q = gate[j][v];
                q = gates_of(to_f32(r[j].v[v]), to_f32(i[j].v[v]), rate_s[cl + v]);
                if (kind[j] == kStart) { q.a = 0.0f; q.beta = 1.0f; q.inv_beta = 0.0f; }
                u[j][v] = q.beta * q.si.s * to_f32(x[j].v[v]);
                H[v] = fmaf(q.a, H[v], u[j][v]);
                A[v] *= q.a;
            }
        }
    }
#pragma unroll
    for (int j = Tc - 1; j >= 0; --j)
        if (kind[j] > kPadding)
#pragma unroll
            for (int v = 0; v < V; ++v) R[v] = gate[j][v].a * (to_f32(g[j].v[v]) + R[v]);
    float A_before[V], H_before[V], A_after[V], R_after[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float Af = A[v], Ab = A[v];
#pragma unroll
        for (int d = 8; d < kWave; d *= 2) {
            const float pA = __shfl_up(Af, d), pH = __shfl_up(H[v], d), nA = __shfl_down(Ab, d), nR = __shfl_down(R[v], d);
            if (lane >= d) {
                H[v] = fmaf(Af, pH, H[v]);
                Af *= pA;
            }
            if (lane < kWave - d) {
                R[v] = fmaf(Ab, nR, R[v]);
                Ab *= nA;
            }
        }
        A_before[v] = __shfl_up(Af, 8);
        H_before[v] = __shfl_up(H[v], 8);
        A_after[v] = __shfl_down(Ab, 8);
        R_after[v] = __shfl_down(R[v], 8);
        if (lane < 8) { A_before[v] = 1.0f; H_before[v] = 0.0f; }
        if (lane >= kWave - 8) {
            A_after[v] = 1.0f;
            R_after[v] = 0.0f;
            A_s[wave][cl + v] = Af;
            H_s[wave][cl + v] = H[v];
        }
        if (lane < 8) R_s[wave][cl + v] = R[v];
    }
    lds_barrier();
    if (wave == 0) {
        const int ch = at.c0 + lane;
        const bool mine = lane < CT && ch < p.C;
        float D = 0.0f, Aw = 1.0f, Rw = 0.0f;
        if (mine) {
            float h = p.T > 0 ? p.states[((int64_t)at.b * p.kept + unit) * p.C + ch] : 0.0f;
            for (int w = 0; w < NW; ++w) {
                carry_s[w][lane] = h;
                h = fmaf(A_s[w][lane], h, H_s[w][lane]);
            }
            for (int w = NW - 1; w >= 0; --w) { Rw = fmaf(A_s[w][lane], Rw, R_s[w][lane]); Aw *= A_s[w][lane]; }
        }
        if constexpr (CHAIN) {
            const int64_t stride = (int64_t)p.sequences * CT;
            Word *own = p.words + (int64_t)at.seq * CT + lane;
            if (at.unit > 0) {
                if (mine) publish(own + at.unit * stride, Aw, Rw);
                D = look_back(own, at.unit - 1, stride, mine);
            } else if (mine) {
                D = p.grad_h_last[(int64_t)at.b * p.C + ch];
            }
            if (mine) publish(own + at.unit * stride, 0.0f, fmaf(Aw, D, Rw));
        } else if (mine && p.grad_h_last) {
            D = p.grad_h_last[(int64_t)at.b * p.C + ch];
        }
        if (mine) {
            for (int w = NW - 1; w >= 0; --w) {
                after_s[w][lane] = D;
                D = fmaf(A_s[w][lane], D, R_s[w][lane]);
            }
            if (p.grad_h_first && unit == 0) p.grad_h_first[(int64_t)at.b * p.C + ch] = D;
        }
    }
    lds_barrier();
    float sum[V], before[Tc][V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        sum[v] = 0.0f;
        float h = fmaf(A_before[v], carry_s[wave][cl + v], H_before[v]);
#pragma unroll
        for (int j = 0; j < Tc; ++j) {
            before[j][v] = h;
            h = fmaf(gate[j][v].a, h, u[j][v]);
        }
    }
    float D[V];
#pragma unroll
    for (int v = 0; v < V; ++v) D[v] = fmaf(A_after[v], after_s[wave][cl + v], R_after[v]);
#pragma unroll
    for (int j = Tc - 1; j >= 0; --j) {
        if (kind[j] == kPast) continue;
        Row<E, VEC> gx, gr, gi;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float dx = 0.0f, dr = 0.0f, di = 0.0f;
            if (kind[j] != kPadding) {
                const Gates &q = gate[j][v];
                const float xv = to_f32(x[j].v[v]), dh = to_f32(g[j].v[v]) + D[v], du = dh * q.beta;
                dx = du * q.si.s;
                di = dx * xv * q.si.c;
                D[v] = q.a * dh;
                const float dL = D[v] * (before[j][v] - q.si.s * xv * q.a * q.inv_beta);       // (a = 0 at a sequence's start)
                const float part = q.sr.s * dL;
                dr = -rate_s[cl + v] * q.sr.c * part;
                sum[v] -= part;
            }
            gx.v[v] = from_f32<E>(dx);
            gr.v[v] = from_f32<E>(dr);
            gi.v[v] = from_f32<E>(di);
        }
        const int64_t row = (int64_t)at.b * p.T + t0 + j;
        gx.store(p.grad_x, row * p.ld_gx + c, left);
        gr.store(p.grad_r, row * p.ld_gr + c, left);
        gi.store(p.grad_i, row * p.ld_gi + c, left);
    }
    // the unit's part of the sum for lam: groups, then waves, in order
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int d = 8; d < kWave; d *= 2) sum[v] += __shfl_xor(sum[v], d);
        if (lane < 8) H_s[wave][cl + v] = sum[v];
    }
    lds_barrier();
    for (int k = threadIdx.x; k < CT; k += NW * kWave) {
        if (at.c0 + k >= p.C) continue;
        float total = 0.0f;
        for (int w = 0; w < NW; ++w) total += H_s[w][k];
        p.lam_part[((int64_t)at.b * p.units + unit) * p.C + at.c0 + k] = total;
    }
}

// grad_lam[c] = decay sigmoid(lam[c]) * sum of the units' parts: 16 runs of each channel side by side, then together, in order.
__global__ __launch_bounds__(1024) void scan_lam_kernel(ScanArgs p, int64_t parts)
{
    __shared__ float run[16][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c = blockIdx.x * kWave + lane;
    float sum = 0.0f;
    if (c < p.C)
        for (int64_t k = wave; k < parts; k += 16) sum += p.lam_part[k * p.C + c];
    run[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || c >= p.C) return;
    for (int w = 1; w < 16; ++w) sum += run[w][lane];
    p.grad_lam[c] = sum * p.decay * sigmoid2(p.lam[c]).s;
}

struct StepArgs {
    int n, C, slots;
    const void *x, *r, *i;
    int64_t ld_x, ld_r, ld_i;
    const float *lam;
    float decay;
    const int32_t *slot;
    const uint8_t *reset;
    const float *h_in;
    float *h_out;
    void *y;
    int64_t ld_y;
};

template <typename E>
__global__ __launch_bounds__(256) void step_kernel(StepArgs p)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (int64_t)p.n * p.C) return;
    const int64_t row = id / p.C;
    const int c = (int)(id % p.C);
    const int64_t at = (int64_t)(p.slot ? min(max(p.slot[row], 0), p.slots - 1) : (int)row) * p.C + c;
    const Gates g = gates_of(to_f32(static_cast<const E *>(p.r)[row * p.ld_r + c]),
                             to_f32(static_cast<const E *>(p.i)[row * p.ld_i + c]), rate_of(p.lam[c], p.decay));
    const float in = g.si.s * to_f32(static_cast<const E *>(p.x)[row * p.ld_x + c]);
    const float h = p.reset && p.reset[row] ? in : fmaf(g.a, p.h_in[at], g.beta * in);
    p.h_out[at] = h;
    static_cast<E *>(p.y)[row * p.ld_y + c] = from_f32<E>(h);
}

bool scan_sizes_ok(int B, int T, int C)
{
    return B >= 0 && T >= 0 && C >= 0 && C < (1 << 24) && (int64_t)B * T < ((int64_t)1 << 30) && (int64_t)B * C < ((int64_t)1 << 31);
}

// How a call is cut, and where things lie in the workspace (the kept states first: they outlive the call).
struct ScanPlan {
    int waves, waves_back, units, units_back, tiles;
    size_t states, aside, words, ticket, lam_part, bytes;
    int64_t n_words;
};

ScanPlan scan_plan(int dtype, int B, int T, int C)
{
    const int V = 16 / element_bytes(dtype), CT = 8 * V, lane = kElements / V, lane_back = kElementsBack / V;
    ScanPlan s{};
    s.waves = waves_for(T, lane);
    s.waves_back = waves_for(T, lane_back);
    auto units = [&](int steps) { return T > 0 ? (T + steps - 1) / steps : 1; };
    s.units = units(s.waves * 8 * lane);
    s.units_back = units(s.waves_back * 8 * lane_back);
    s.tiles = (C + CT - 1) / CT;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    s.states = take((size_t)B * s.units_back * C * sizeof(float));
    s.aside = take((size_t)B * C * sizeof(float));
    s.n_words = s.units_back > 1 ? (int64_t)s.units_back * B * s.tiles * CT : 0;       // never fewer units than forward
    s.words = take((size_t)s.n_words * sizeof(Word));
    s.ticket = take(sizeof(unsigned));
    s.lam_part = take((size_t)B * s.units_back * C * sizeof(float));
    s.bytes = at;
    return s;
}

bool positive(float v) { return std::isfinite(v) && v > 0.0f; }

// Checks that the forward and the backward call have in common.
int scan_check(int dtype, int B, int T, int C, float decay, const void *workspace, size_t workspace_bytes)
{
    if (!known_dtype(dtype)) return MARL_ERR_BAD_DTYPE;
    if (!scan_sizes_ok(B, T, C)) return MARL_ERR_BAD_DIM;
    if (!positive(decay)) return MARL_ERR_BAD_ARG;
    if (workspace_bytes < scan_plan(dtype, B, T, C).bytes) return MARL_ERR_BAD_DIM;
    if (!workspace && workspace_bytes) return MARL_ERR_NULL;
    return aligned_to(workspace, 256) ? MARL_OK : MARL_ERR_BAD_ARG;
}

unsigned blocks_of(int64_t n) { return (unsigned)((n + 255) / 256); }

// Rows can be read 16 bytes at a time: everything is a multiple of 16 bytes apart.
bool rows_of_sixteen(int dtype, int C, std::initializer_list<const void *> pointers, std::initializer_list<int64_t> strides)
{
    const int V = 16 / element_bytes(dtype);
    bool ok = C % V == 0;
    for (const void *p : pointers) ok = ok && aligned_to(p, 16);
    for (int64_t ld : strides) ok = ok && ld % V == 0;
    return ok;
}

// Calls f(std::integral_constant<int, waves>).
template <typename F>
int with_waves(int waves, F &&f)
{
    switch (waves) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 4: return f(std::integral_constant<int, 4>{});
    default: return f(std::integral_constant<int, kMostWaves>{});
    }
}

template <bool BACK, typename E, bool VEC, int NW, bool CHAIN>
int launch_scan(const ScanArgs &p, hipStream_t stream)
{
    const dim3 grid((unsigned)(p.units * p.sequences)), block(NW * kWave);
    if constexpr (BACK) hipLaunchKernelGGL((scan_grad_kernel<E, VEC, NW, CHAIN>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((scan_kernel<E, VEC, NW, CHAIN>), grid, block, 0, stream, p);
    return launched(BACK ? "linear scan gradient" : "linear scan");
}

// One workgroup per unit; with more than one unit in a sequence they hand the state on.
template <bool BACK>
int run_scan(int dtype, ScanArgs p, const ScanPlan &s, char *workspace, bool vec, hipStream_t stream)
{
    p.tiles = s.tiles;
    if ((int64_t)p.B * s.tiles * (BACK ? s.units_back : s.units) >= ((int64_t)1 << 31)) return MARL_ERR_BAD_DIM;
    p.sequences = p.B * s.tiles;
    p.units = BACK ? s.units_back : s.units;
    p.states = reinterpret_cast<float *>(workspace + s.states);
    p.kept = s.units_back;
    p.keep = s.waves_back * 8 * kElementsBack / (16 / element_bytes(dtype));
    p.lam_part = reinterpret_cast<float *>(workspace + s.lam_part);
    p.words = reinterpret_cast<Word *>(workspace + s.words);
    p.ticket = reinterpret_cast<unsigned *>(workspace + s.ticket);
    if (p.units > 1) {
        float *aside = reinterpret_cast<float *>(workspace + s.aside);
        const int64_t n_states = (int64_t)p.B * p.C, n_words = (int64_t)p.units * p.sequences * 128 / element_bytes(dtype);
        hipLaunchKernelGGL(scan_begin_kernel, dim3(blocks_of(n_words > n_states ? n_words : n_states)), dim3(256), 0, stream, p.words, n_words, p.ticket,
                           BACK ? p.grad_h_last : p.h_first, aside, n_states);
        (BACK ? p.grad_h_last : p.h_first) = aside;
        return with_dtype(dtype, [&](auto e) {
            return vec ? launch_scan<BACK, decltype(e), true, kMostWaves, true>(p, stream) : launch_scan<BACK, decltype(e), false, kMostWaves, true>(p, stream);
        });
    }
    return with_dtype(dtype, [&](auto e) {
        return with_waves(BACK ? s.waves_back : s.waves, [&](auto waves) {
            return vec ? launch_scan<BACK, decltype(e), true, decltype(waves)::value, false>(p, stream)
                       : launch_scan<BACK, decltype(e), false, decltype(waves)::value, false>(p, stream);
        });
    });
}

}  // namespace
}  // namespace marl

using namespace marl;

extern "C" {

int marl_linear_scan_workspace_bytes(int32_t dtype, int32_t B, int32_t T, int32_t C, size_t *bytes)
{
    if (!bytes) return MARL_ERR_NULL;
    if (!known_dtype(dtype)) return MARL_ERR_BAD_DTYPE;
    if (!scan_sizes_ok(B, T, C)) return MARL_ERR_BAD_DIM;
    *bytes = scan_plan(dtype, B, T, C).bytes;
    return MARL_OK;
}

int marl_linear_scan(int32_t dtype, int32_t B, int32_t T, int32_t C, const void *x, int64_t ld_x, const void *r,
                     int64_t ld_r, const void *i, int64_t ld_i, const float *lam, float decay, const uint8_t *reset,
                     const uint8_t *filled, const float *h_first, void *y, int64_t ld_y, float *h_last,
                     void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const int rc = scan_check(dtype, B, T, C, decay, workspace, workspace_bytes);
    if (rc) return rc;
    if (B == 0 || C == 0) return MARL_OK;
    if (!lam || (T > 0 && (!x || !r || !i || !y))) return MARL_ERR_NULL;
    if (ld_x < C || ld_r < C || ld_i < C || ld_y < C) return MARL_ERR_BAD_DIM;
    if (T > 0 && (y == x || y == r || y == i)) return MARL_ERR_BAD_ARG;
    ScanArgs p{};
    p.B = B; p.T = T; p.C = C;
    p.x = x; p.r = r; p.i = i; p.ld_x = ld_x; p.ld_r = ld_r; p.ld_i = ld_i;
    p.lam = lam; p.decay = decay; p.reset = reset; p.filled = filled; p.h_first = h_first;
    p.y = y; p.ld_y = ld_y; p.h_last = h_last;
    const bool vec = rows_of_sixteen(dtype, C, {x, r, i, y}, {ld_x, ld_r, ld_i, ld_y});
    return run_scan<false>(dtype, p, scan_plan(dtype, B, T, C), static_cast<char *>(workspace), vec, static_cast<hipStream_t>(hip_stream));
}

int marl_linear_scan_grad(int32_t dtype, int32_t B, int32_t T, int32_t C, const void *x, int64_t ld_x, const void *r,
                          int64_t ld_r, const void *i, int64_t ld_i, const float *lam, float decay,
                          const uint8_t *reset, const uint8_t *filled, const void *grad_y, int64_t ld_gy,
                          const float *grad_h_last, void *workspace, size_t workspace_bytes, void *grad_x,
                          int64_t ld_gx, void *grad_r, int64_t ld_gr, void *grad_i, int64_t ld_gi, float *grad_lam,
                          float *grad_h_first, void *hip_stream)
{
    const int rc = scan_check(dtype, B, T, C, decay, workspace, workspace_bytes);
    if (rc) return rc;
    if (C == 0) return MARL_OK;
    if (!lam || !grad_lam || (B > 0 && T > 0 && (!x || !r || !i || !grad_y || !grad_x || !grad_r || !grad_i))) return MARL_ERR_NULL;
    if (ld_x < C || ld_r < C || ld_i < C || ld_gy < C || ld_gx < C || ld_gr < C || ld_gi < C) return MARL_ERR_BAD_DIM;
    const void *in[4] = {x, r, i, grad_y}, *out[3] = {grad_x, grad_r, grad_i};
    for (int k = 0; k < 3; ++k) {
        for (const void *v : in)
            if (v && out[k] == v) return MARL_ERR_BAD_ARG;
        if (out[k] && out[k] == out[(k + 1) % 3]) return MARL_ERR_BAD_ARG;
    }
    ScanArgs p{};
    p.B = B; p.T = T; p.C = C;
    p.x = x; p.r = r; p.i = i; p.ld_x = ld_x; p.ld_r = ld_r; p.ld_i = ld_i;
    p.lam = lam; p.decay = decay; p.reset = reset; p.filled = filled;
    p.grad_y = grad_y; p.ld_gy = ld_gy; p.grad_h_last = grad_h_last;
    p.grad_x = grad_x; p.grad_r = grad_r; p.grad_i = grad_i; p.ld_gx = ld_gx; p.ld_gr = ld_gr; p.ld_gi = ld_gi;
    p.grad_lam = grad_lam; p.grad_h_first = grad_h_first;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const ScanPlan s = scan_plan(dtype, B, T, C);
    if (B > 0) {
        const bool vec = rows_of_sixteen(dtype, C, {x, r, i, grad_y, grad_x, grad_r, grad_i}, {ld_x, ld_r, ld_i, ld_gy, ld_gx, ld_gr, ld_gi});
        const int status = run_scan<true>(dtype, p, s, static_cast<char *>(workspace), vec, stream);
        if (status) return status;
        p.lam_part = reinterpret_cast<float *>(static_cast<char *>(workspace) + s.lam_part);
    }
    hipLaunchKernelGGL(scan_lam_kernel, dim3((unsigned)((C + kWave - 1) / kWave)), dim3(1024), 0, stream, p, (int64_t)B * s.units_back);
    return launched("linear scan gradient");
}

int marl_linear_step(int32_t dtype, int32_t n, int32_t C, const void *x, int64_t ld_x, const void *r, int64_t ld_r,
                     const void *i, int64_t ld_i, const float *lam, float decay, const int32_t *slot, int32_t slots,
                     const uint8_t *reset, const float *h_in, float *h_out, void *y, int64_t ld_y, void *hip_stream)
{
    if (!known_dtype(dtype)) return MARL_ERR_BAD_DTYPE;
    if (n < 0 || C < 0 || C >= (1 << 24) || slots < 1 || (!slot && n > slots) || (int64_t)n * C >= ((int64_t)1 << 38)) return MARL_ERR_BAD_DIM;
    if (!positive(decay)) return MARL_ERR_BAD_ARG;
    if (n == 0 || C == 0) return MARL_OK;
    if (!x || !r || !i || !lam || !h_in || !h_out || !y) return MARL_ERR_NULL;
    if (ld_x < C || ld_r < C || ld_i < C || ld_y < C) return MARL_ERR_BAD_DIM;
    if (y == x || y == r || y == i) return MARL_ERR_BAD_ARG;
    const StepArgs p{n, C, slots, x, r, i, ld_x, ld_r, ld_i, lam, decay, slot, reset, h_in, h_out, y, ld_y};
    return with_dtype(dtype, [&](auto e) {
        hipLaunchKernelGGL((step_kernel<decltype(e)>), dim3(blocks_of((int64_t)n * C)), dim3(256), 0, static_cast<hipStream_t>(hip_stream), p);
        return launched("linear step");
    });
}

}  // extern "C"
