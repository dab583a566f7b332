// Gated linear recurrence: h[t] = a[t] h[t-1] + beta[t] sigmoid(i[t]) x[t], its backward pass and its form for one step.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "device_math.h"
#include "operator_types.h"

namespace marl {
namespace {

// The shape of the work.  A workgroup (a "unit") takes 64 channels over a span of steps.  A lane takes four bytes of a row
// (V channels) and Tc steps that follow one another; lanes of one row lie side by side, and the wave holds V rows' worth of
// lanes ("groups"), then waves, then units, which follow one another in time.  What a stretch of steps does to the
// state is h -> A h + H, and stretches compose: a lane composes its own steps, the two groups of 16-bit types compose by lane
// exchange, the waves through shared memory, and units through memory (see look_back).  The inputs are read once and stay
// in registers until the state at the unit's start is known.
// Narrow and long units: the number of units of one sequence in flight, which is what look_back walks over, is small.  Fewer than 64
// channels leave lanes without work: 64 x 4000 steps fp32 take 114 us there and back with 16 channels, 179 us with 64.  Four
// bytes a lane rather than sixteen: with eight channels a lane the lane exchanges were eight per element of the backward pass.
constexpr int kChannels = 64;
template <typename E> constexpr int kWide = 4 / (int)sizeof(E);            // V: channels of a lane, groups of a wave
constexpr int kSteps = 16;                                                 // Tc forward
template <typename E> constexpr int kStepsBack = 16 / kWide<E>;            // Tc backward: 16 elements, of which more is kept

// Most waves of a unit, and the waves that T needs.  The backward pass keeps seven values of each element: four waves of 168
// registers, three units on a compute unit.
constexpr int kMostWaves = 8, kMostWavesBack = 4;
inline int waves_for(int T, int wave_steps, int most)
{
    int w = 1;
    while (w < most && w * wave_steps < T) w *= 2;
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
    float *states;                     // [B, kept, C] state before each 2^keep_log-th step
    int keep_log, kept;
    unsigned *ticket;                  // order in which units begin
    Word *words;                       // [units, sequences, 64]
    // backward pass
    const void *grad_y;
    int64_t ld_gy;
    const float *grad_h_last;
    void *grad_x, *grad_r, *grad_i;
    int64_t ld_gx, ld_gr, ld_gi;
    float *lam_part;                   // [B units, C]
    float *grad_lam, *grad_h_first;
};

// decay log(1 + e^lam).  The rounding of 1 + e is undone by the quotient (Kahan): log(u) e / (u - 1) with u = 1 + e as rounded.
__device__ __forceinline__ float rate_of(float lam, float decay)
{
    const float e = __builtin_amdgcn_exp2f(kLog2e * lam), u = 1.0f + e, d = u - 1.0f;
    const float soft = d == 0.0f ? e : __builtin_amdgcn_logf(u) * 0.69314718f * (e * __builtin_amdgcn_rcpf(d));
    return decay * (lam > 20.0f ? lam : soft);                 // (above 20 the difference is below half a step)
}

// sigmoid(v) and its complement, each to fp32 accuracy at both ends, from e^-v, which ends where they are below fp32 anyway.  NaN stays NaN.
struct Sigmoid { float s, c; };
__device__ __forceinline__ float odds_against(float v) { return __builtin_elementwise_minimum(__builtin_amdgcn_exp2f(-kLog2e * v), 1e37f); }
__device__ __forceinline__ Sigmoid sigmoid_of_odds(float e)
{
    const float s = __builtin_amdgcn_rcpf(1.0f + e);
    return {s, e * s};
}
__device__ __forceinline__ Sigmoid sigmoid2(float v) { return sigmoid_of_odds(odds_against(v)); }

// The decay of a step: a = 2^e with e = -log2(e) rate sigmoid(r) <= 0, and beta^2 = 1 - a^2.  Near 0 the difference would cancel:
// there -2 a sinh(e ln 2) by its series up to the seventh power, whose next term is below 2^-26 of it.  `rate2` is -log2(e) rate.
// `start` is 0, or -200 where a sequence starts: then a is 0 and beta 1.
struct Decay { float a, om; };
__device__ __forceinline__ Decay decay_of(float s_r, float rate2, float start)
{
    constexpr double l = 0.69314718055994530942, l3 = l * l * l, l5 = l3 * l * l, l7 = l5 * l * l;
    const float e = fmaf(rate2, s_r, start), a = __builtin_amdgcn_exp2f(e), q = e * e;
    float p = fmaf(q, (float)(-2.0 * l7 / 5040.0), (float)(-2.0 * l5 / 120.0));
    p = fmaf(q, p, (float)(-2.0 * l3 / 6.0));
    p = fmaf(q, p, (float)(-2.0 * l));
    const float near = a * (e * p), far = fmaf(-a, a, 1.0f);
    return {a, e > -0.72f ? near : far};
}

// What one step does forward: h -> a h + u.
struct Step { float a, u; };
__device__ __forceinline__ Step step_of(float x, float r, float i, float rate2, float start)
{
    const Decay d = decay_of(sigmoidf_fast(r), rate2, start);
    return {d.a, __builtin_amdgcn_sqrtf(d.om) * (x * sigmoidf_fast(i))};
}

// And what its gradients need: dx = dh m, di = dh n, dL = a dh (h before - q), dr = -rate (1 - s) s dL.  odds: e^-r, from which both s and
// 1 - s come (1 - s from s would cancel where the gate is open: at r = 10 two digits of it were left).
struct StepBack { float a, u, q, m, n, odds; };
__device__ __forceinline__ StepBack step_back_of(float x, float r, float i, float rate2, float start)
{
    const Sigmoid si = sigmoid2(i);
    float odds = odds_against(r);
    const Decay d = decay_of(sigmoid_of_odds(odds).s, rate2, start);
    asm("" : "+v"(odds));                                              // s is formed again when it is wanted, or it is kept too, and registers spill
    const float inv = __builtin_amdgcn_rsqf(fmaxf(d.om, 1e-30f));      // a gate that is shut has om = 0: beta 0, and no infinity
    const float beta = d.om * inv, in = si.s * x, u = beta * in;
    return {d.a, u, d.a * inv * in, beta * si.s, u * si.c, odds};
}

// All bits or none, after bit j of `bits`.
__device__ __forceinline__ uint32_t all_of(unsigned bits, int j) { return (uint32_t)((int)(bits << (31 - j)) >> 31); }
__device__ __forceinline__ float start_of(unsigned start, int j) { return __uint_as_float(all_of(start, j) & 0xc3480000u); }
// v, or 0 at step j if its bit of `start` is set: a product with a = 0 would let an infinity or NaN of the sequence before through.
__device__ __forceinline__ float unless_start(float v, unsigned start, int j) { return __uint_as_float(__float_as_uint(v) & ~all_of(start, j)); }
// The same where stretches meet: what one does to the state, and what two do that follow one another.  A = 0 says that a sequence starts in
// the stretch, and nothing of before is left, infinity and NaN included.  A product of decays alone never says so: it ends at
// the smallest normal number, which leaves less than 2^-26 of a state below 2^100, and through which what is not finite stays so.  (By its bits: a product is
// not negative, and NaN lies above all.)
__device__ __forceinline__ float decayed(float A) { return __uint_as_float(max(__float_as_uint(A), 0x00800000u)); }
__device__ __forceinline__ float follow(float A, float h, float H) { return A == 0.0f ? H : fmaf(A, h, H); }
__device__ __forceinline__ float both(float A, float B) { return A == 0.0f || B == 0.0f ? 0.0f : decayed(A * B); }

// Four bytes of a row.  PAIRS: they lie at a multiple of four bytes and there is no odd channel at the end.
// Held as one word: as a pair of 16-bit values the compiler gave each a register of its own wherever branches meet.
template <typename E, bool PAIRS>
struct Row {
    static constexpr int V = kWide<E>;
    typedef E Vec __attribute__((ext_vector_type(V)));
    uint32_t bits;
    __device__ __forceinline__ void get(float (&f)[V]) const
    {
        uint32_t b = bits;
        asm("" : "+v"(b));
        const Vec v = __builtin_bit_cast(Vec, b);
#pragma unroll
        for (int k = 0; k < V; ++k) f[k] = to_f32(v[k]);
    }
    // Without m the row is zeros; a gate's row is -infinity, a gate that is shut: the step does nothing to the state.
    __device__ __forceinline__ void keep(uint32_t m) { bits &= m; }
    __device__ __forceinline__ void keep_or_shut(uint32_t m)
    {
        constexpr uint32_t shut = sizeof(E) == 4 ? 0xff800000u : std::is_same<E, __bf16>::value ? 0xff80ff80u : 0xfc00fc00u;
        bits = (bits & m) | (shut & ~m);
    }
    __device__ __forceinline__ void set(const float (&f)[V])
    {
        Vec v;
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = from_f32<E>(f[k]);
        bits = __builtin_bit_cast(uint32_t, v);
    }
};

// A wave's rows of one array: the first one's address is the same for the wave, a lane adds its group's rows and its
// channels, and a step adds a distance that is the same for all: no vector arithmetic per access.  reach: steps behind
// the first that exist; loads of later ones read the last (and are dropped), stores are left out.
template <typename E, bool PAIRS>
struct Strip {
    static constexpr int V = kWide<E>;
    char *base;
    int64_t step;                      // bytes
    uint32_t lane;                     // bytes
    int c;                             // element of the row
    __device__ __forceinline__ Strip(const void *p, int64_t ld, int64_t row, int c0, int cl, int rows_down)
        : base(static_cast<char *>(const_cast<void *>(p)) + (row * ld + c0) * (int)sizeof(E)), step(ld * (int)sizeof(E)),
          lane((uint32_t)rows_down * (uint32_t)step + (uint32_t)cl * (uint32_t)sizeof(E)), c(cl) {}
    // the row in hand, and on to the next one (in turn: all rows' addresses at once do not fit the scalar registers)
    __device__ __forceinline__ void load(Row<E, PAIRS> &r, int left)
    {
        read(r, base + lane, left);
        base += step;
    }
    __device__ __forceinline__ void load_within(Row<E, PAIRS> &r, int t, int reach, int left) const
    {
        read(r, base + (int64_t)min(t, reach) * step + (uint32_t)c * (uint32_t)sizeof(E), left);
    }
    __device__ __forceinline__ void read(Row<E, PAIRS> &r, const char *at, int left) const
    {
        if constexpr (PAIRS) {
            r.bits = *reinterpret_cast<const uint32_t *>(at);
        } else {
            typename Row<E, PAIRS>::Vec v;
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = k < left ? reinterpret_cast<const E *>(at)[k] : (E)0.0f;
            r.bits = __builtin_bit_cast(uint32_t, v);
        }
    }
    __device__ __forceinline__ void store(const Row<E, PAIRS> &r, int left) const
    {
        char *at = base + lane;
        if constexpr (PAIRS) {
            *reinterpret_cast<uint32_t *>(at) = r.bits;
        } else {
            const typename Row<E, PAIRS>::Vec v = __builtin_bit_cast(typename Row<E, PAIRS>::Vec, r.bits);
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k < left) reinterpret_cast<E *>(at)[k] = v[k];
        }
    }
};

__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Which of the N steps from t0 on (N <= 32, the same for the whole wave) exist, are filled, start a sequence: a bit each.
struct Steps { unsigned exist, filled, start; };
template <int N>
__device__ __forceinline__ Steps steps_at(const ScanArgs &p, int64_t b, int t0)
{
    const int lane = threadIdx.x % kWave, t = t0 + lane;
    const bool exist = lane < N && t < p.T;
    const int64_t row = b * p.T + (exist ? t : 0);
    const bool filled = exist && (!p.filled || p.filled[row]), start = filled && p.reset && p.reset[row];
    return {(unsigned)__ballot(exist), (unsigned)__ballot(filled), (unsigned)__ballot(start)};
}

__device__ __forceinline__ Word word_of(float A, float H)
{
    return (Word)(__float_as_uint(A) | 0x80000000u) << 32 | __float_as_uint(H);
}
__device__ __forceinline__ void publish(Word *at, float A, float H) { __hip_atomic_store(at, word_of(A, H), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ Word peek(const Word *at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__device__ __forceinline__ float word_A(Word w) { return __uint_as_float((unsigned)(w >> 32) & 0x7fffffffu); }
__device__ __forceinline__ float word_H(Word w) { return __uint_as_float((unsigned)w); }

// The state at the start of a unit, a lane per channel.  Units publish (A, H) of their own steps at once, without waiting
// for anything, and (0, h) of the state behind them when they know it; A = 0 says that nothing before matters.  Walking
// backwards from unit `before` over whichever is there, `stride` words apart, until A = 0; the first unit publishes (0, h) alone.
// What was met is then applied in the order of time, one unit after the other, as each unit does for the state that it publishes:
// the same sums in the same order whichever of the two words was there, so that timing does not change a bit.  The last of the
// kDeep words that there is room for has to be (0, h).  A unit waits only for units whose tickets are lower, and they began before it:
// each wait ends.
template <int kAtOnce, int kDeep>
__device__ __forceinline__ float look_back(const Word *words, int before, int64_t stride, bool mine, Word (&held)[kDeep][kChannels])
{
    const int lane = threadIdx.x % kWave;
    bool open = mine;
    int n = 0;
    for (int k = before; k >= 0 && __any(open); k -= kAtOnce) {
        Word w[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) w[j] = open && k - j >= 0 ? peek(words + (int64_t)(k - j) * stride + lane) : 0;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (k - j < 0 || !__any(open)) break;
            const bool last = n == kDeep - 1;
            while (__any(open && (w[j] == 0 || (last && word_A(w[j]) != 0.0f)))) {
                __builtin_amdgcn_s_sleep(1);
                if (open) w[j] = peek(words + (int64_t)(k - j) * stride + lane);
            }
            held[n++][lane] = open ? w[j] : 0;
            open = open && word_A(w[j]) != 0.0f;
        }
    }
    float h = 0.0f;
#pragma unroll kAtOnce
    while (n > 0) {
        const Word w = held[--n][lane];
        h = follow(word_A(w), h, word_H(w));
    }
    return h;
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
template <bool CHAIN>
__device__ __forceinline__ Place place_of(const ScanArgs &p, int *shared)
{
    int id = blockIdx.x;
    if constexpr (CHAIN) {
        if (threadIdx.x == 0) *shared = (int)atomicAdd(p.ticket, 1u);
        lds_barrier();
        id = __builtin_amdgcn_readfirstlane(*shared);
    }
    const int seq = id % p.sequences;
    return {seq, id / p.sequences, seq / p.tiles, seq % p.tiles * kChannels};
}

// Forward.  Every input is read once and y written once.  34 instructions an element, six of them transcendental, but waves wait 53 to 55 %
// of their cycles: a unit's loads all stand at its start, and what follows them is a chain through shared memory and the units before.
// 40001 x 1024 bf16 takes 86 us with its small launch (3.8 TB/s), 4 x 16384 x 2048 bf16 225 us (4.8 TB/s; a large copy reaches 5.25); 320 x 120 x 64
// fp32, one unit a sequence, 10 us.
template <typename E, bool PAIRS, int NW, bool CHAIN>
__global__ __launch_bounds__(NW * kWave, 4) void scan_kernel(ScanArgs p)
{
    constexpr int V = kWide<E>, Tc = kSteps, kWaveSteps = V * Tc, kAll = (int)((1ull << kWaveSteps) - 1);
    __shared__ float rate_s[kChannels], A_s[NW][kChannels], H_s[NW][kChannels], carry_s[NW][kChannels];
    __shared__ int id_s;
    __shared__ Word held_s[CHAIN ? 64 : 1][kChannels];
    const Place at = place_of<CHAIN>(p, &id_s);
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), group = lane / (kWave / V), cl = lane % (kWave / V) * V;
    const int c = at.c0 + cl, left = p.C - c, first = at.unit * (NW * kWaveSteps), tw = first + wave * kWaveSteps;
    const Steps steps = steps_at<kWaveSteps>(p, at.b, tw);
    const unsigned exist = steps.exist >> (group * Tc), filled = steps.filled >> (group * Tc), start = steps.start >> (group * Tc);
    const int64_t row0 = (int64_t)at.b * p.T + tw;
    const int down = group * Tc;
    Row<E, PAIRS> x[Tc], r[Tc], i[Tc];
    if (steps.filled && left > 0) {
        Strip<E, PAIRS> sx(p.x, p.ld_x, row0, at.c0, cl, down), sr(p.r, p.ld_r, row0, at.c0, cl, down), si(p.i, p.ld_i, row0, at.c0, cl, down);
        if (steps.exist == (unsigned)kAll) {
#pragma unroll
            for (int j = 0; j < Tc; ++j) {
                __builtin_amdgcn_sched_barrier(0);
                sr.load(r[j], left);
                si.load(i[j], left);
                sx.load(x[j], left);
            }
        } else {
#pragma unroll
            for (int j = 0; j < Tc; ++j) {
                __builtin_amdgcn_sched_barrier(0);
                sr.load_within(r[j], down + j, p.T - 1 - tw, left);
                si.load_within(i[j], down + j, p.T - 1 - tw, left);
                sx.load_within(x[j], down + j, p.T - 1 - tw, left);
            }
        }
    }
    for (int k = threadIdx.x; k < kChannels; k += NW * kWave) rate_s[k] = at.c0 + k < p.C ? rate_of(p.lam[at.c0 + k], p.decay) : 0.0f;
    lds_barrier();
    float rate2[V];
#pragma unroll
    for (int v = 0; v < V; ++v) rate2[v] = -kLog2e * rate_s[cl + v];
    float a[Tc][V], u[Tc][V], A[V], H[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { A[v] = 1.0f; H[v] = 0.0f; }
    if (steps.filled != (unsigned)kAll) {
#pragma unroll
        for (int j = 0; j < Tc; ++j) {
            const uint32_t m = all_of(filled, j);
            x[j].keep(m);
            i[j].keep(m);
            r[j].keep_or_shut(m);
        }
    }
    if (steps.start) {                                         // a start has no decay of its own: its gate is not looked at
#pragma unroll
        for (int j = 0; j < Tc; ++j) r[j].keep(~all_of(start, j));
    }
#pragma unroll
    for (int j = 0; j < Tc; ++j) {
        __builtin_amdgcn_sched_barrier(0);                             // a step at a time, or registers run out
        const float begins = start_of(start, j);
        float xv[V], rv[V], iv[V];
        x[j].get(xv);
        r[j].get(rv);
        i[j].get(iv);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Step s = step_of(xv[v], rv[v], iv[v], rate2[v], begins);
            a[j][v] = s.a;
            u[j][v] = s.u;
            H[v] = fmaf(s.a, unless_start(H[v], start, j), s.u);
            A[v] *= s.a;
        }
    }
    const bool cut = (start & ((1u << Tc) - 1)) != 0;          // nothing passes the lane's steps, whatever their other decays are
    // what the group before this one does, and the wave
    float A_before[V], H_before[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        A[v] = cut ? 0.0f : decayed(A[v]);
        A_before[v] = 1.0f;
        H_before[v] = 0.0f;
        if constexpr (V == 2) {
            const float pA = __shfl_xor(A[v], 32), pH = __shfl_xor(H[v], 32);
            if (group == 1) {
                A_before[v] = pA;
                H_before[v] = pH;
                H[v] = follow(A[v], pH, H[v]);
                A[v] = both(A[v], pA);
            }
        }
        if (group == V - 1) { A_s[wave][cl + v] = A[v]; H_s[wave][cl + v] = H[v]; }
    }
    lds_barrier();
    if (wave == 0) {
        const int ch = at.c0 + lane;
        const bool mine = ch < p.C;
        float Aw = 1.0f, Hw = 0.0f;
        for (int w = 0; w < NW; ++w) { Hw = follow(A_s[w][lane], Hw, H_s[w][lane]); Aw = both(Aw, A_s[w][lane]); }
        float h = 0.0f;
        if constexpr (CHAIN) {
            const int64_t stride = (int64_t)p.sequences * kChannels;
            Word *own = p.words + (int64_t)at.seq * kChannels;
            if (at.unit > 0) {
                if (mine) publish(own + at.unit * stride + lane, Aw, Hw);
                h = look_back<4>(own, at.unit - 1, stride, mine, held_s);
            } else if (mine) {
                h = p.h_first[(int64_t)at.b * p.C + ch];
            }
            if (mine) publish(own + at.unit * stride + lane, 0.0f, follow(Aw, h, Hw));
        } else if (mine && p.h_first) {
            h = p.h_first[(int64_t)at.b * p.C + ch];
        }
        for (int w = 0; w < NW; ++w) {
            carry_s[w][lane] = h;
            const int t = first + w * kWaveSteps;
            if (mine && t < p.T && (t & ((1 << p.keep_log) - 1)) == 0) p.states[((int64_t)at.b * p.kept + (t >> p.keep_log)) * p.C + ch] = h;
            h = follow(A_s[w][lane], h, H_s[w][lane]);
        }
        if (mine && p.h_last && at.unit == p.units - 1) p.h_last[(int64_t)at.b * p.C + ch] = h;
    }
    lds_barrier();
    if (left <= 0) return;
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = follow(A_before[v], carry_s[wave][cl + v], H_before[v]);
    Strip<E, PAIRS> sy(p.y, p.ld_y, row0, at.c0, cl, down);
    auto put = [&](auto whole) {                               // whole: every step exists and counts, and none starts a sequence
#pragma unroll
        for (int j = 0; j < Tc; ++j) {
            __builtin_amdgcn_sched_barrier(0);
            Row<E, PAIRS> y;
            float out[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                h[v] = fmaf(a[j][v], whole ? h[v] : unless_start(h[v], start, j), u[j][v]);
                out[v] = h[v];
            }
            y.set(out);
            if (!whole) y.keep(all_of(filled, j));
            if (whole || (exist >> j & 1)) sy.store(y, left);
            sy.base += sy.step;
        }
    };
    if (steps.filled == (unsigned)kAll && !steps.start) put(std::true_type{});
    else put(std::false_type{});
}

// Backward pass.  D[t] = a[t] dL/dh[t] is what reaches h[t-1]: D[t] = a[t] (grad_y[t] + D[t+1]), the same kind of chain
// backwards in time.  h is formed again inside the unit from the state kept at its start.  69 instructions an element and three waves
// on a SIMD, which wait 56 % of their cycles: 4 x 16384 x 2048 bf16 takes 457 us with its small launches (4.1 TB/s), 320 x 120 x 64 fp32 22 us.
template <typename E, bool PAIRS, int NW, bool CHAIN>
__global__ __launch_bounds__(NW * kWave, 3) void scan_grad_kernel(ScanArgs p)
{
    constexpr int V = kWide<E>, Tc = kStepsBack<E>, kWaveSteps = V * Tc, kAll = (1 << kWaveSteps) - 1;
    __shared__ float rate_s[kChannels], A_s[NW][kChannels], H_s[NW][kChannels], R_s[NW][kChannels], carry_s[NW][kChannels], after_s[NW][kChannels];
    __shared__ int id_s;
    __shared__ Word held_s[CHAIN ? 32 : 1][kChannels];          // (three units on a compute unit: 53 KB each)
    __shared__ uint32_t grad_s[CHAIN ? Tc : 1][NW * kWave];    // grad_y during look_back, for whose registers four spilled otherwise
    const Place at = place_of<CHAIN>(p, &id_s);
    const int unit = p.units - 1 - at.unit;                    // the last steps first
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), group = lane / (kWave / V), cl = lane % (kWave / V) * V;
    const int c = at.c0 + cl, left = p.C - c, tw = (unit * NW + wave) * kWaveSteps;
    const Steps steps = steps_at<kWaveSteps>(p, at.b, tw);
    const unsigned exist = steps.exist >> (group * Tc), filled = steps.filled >> (group * Tc), start = steps.start >> (group * Tc);
    const int64_t row0 = (int64_t)at.b * p.T + tw;
    const int down = group * Tc;
    Row<E, PAIRS> x[Tc], r[Tc], i[Tc], g[Tc];
    if (steps.filled && left > 0) {
        Strip<E, PAIRS> sx(p.x, p.ld_x, row0, at.c0, cl, down), sr(p.r, p.ld_r, row0, at.c0, cl, down), si(p.i, p.ld_i, row0, at.c0, cl, down),
            sg(p.grad_y, p.ld_gy, row0, at.c0, cl, down);
        if (steps.exist == (unsigned)kAll) {
#pragma unroll
            for (int j = 0; j < Tc; ++j) {
                __builtin_amdgcn_sched_barrier(0);
                sr.load(r[j], left);
                si.load(i[j], left);
                sx.load(x[j], left);
                sg.load(g[j], left);
            }
        } else {
#pragma unroll
            for (int j = 0; j < Tc; ++j) {
                __builtin_amdgcn_sched_barrier(0);
                sr.load_within(r[j], down + j, p.T - 1 - tw, left);
                si.load_within(i[j], down + j, p.T - 1 - tw, left);
                sx.load_within(x[j], down + j, p.T - 1 - tw, left);
                sg.load_within(g[j], down + j, p.T - 1 - tw, left);
            }
        }
    }
    for (int k = threadIdx.x; k < kChannels; k += NW * kWave) rate_s[k] = at.c0 + k < p.C ? rate_of(p.lam[at.c0 + k], p.decay) : 0.0f;
    lds_barrier();
    float rate[V];
#pragma unroll
    for (int v = 0; v < V; ++v) rate[v] = rate_s[cl + v];
    StepBack q[Tc][V];
    float A[V], H[V], R[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { A[v] = 1.0f; H[v] = 0.0f; R[v] = 0.0f; }
    if (steps.filled != (unsigned)kAll) {
#pragma unroll
        for (int j = 0; j < Tc; ++j) {
            const uint32_t m = all_of(filled, j);
            x[j].keep(m);
            i[j].keep(m);
            g[j].keep(m);
            r[j].keep_or_shut(m);
        }
    }
    if (steps.start) {                                         // a start has no decay of its own: its gate is not looked at
#pragma unroll
        for (int j = 0; j < Tc; ++j) r[j].keep(~all_of(start, j));
    }
#pragma unroll
    for (int j = 0; j < Tc; ++j) {
        __builtin_amdgcn_sched_barrier(0);                             // a step at a time, or registers run out
        const float begins = start_of(start, j);
        float xv[V], rv[V], iv[V];
        x[j].get(xv);
        r[j].get(rv);
        i[j].get(iv);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            q[j][v] = step_back_of(xv[v], rv[v], iv[v], -kLog2e * rate[v], begins);
            H[v] = fmaf(q[j][v].a, unless_start(H[v], start, j), q[j][v].u);
            A[v] *= q[j][v].a;
        }
    }
#pragma unroll
    for (int j = Tc - 1; j >= 0; --j) {
        float gv[V];
        g[j].get(gv);
#pragma unroll
        for (int v = 0; v < V; ++v) R[v] = unless_start(q[j][v].a * (gv[v] + R[v]), start, j);
    }
    if constexpr (CHAIN) {
#pragma unroll
        for (int j = 0; j < Tc; ++j) grad_s[j][threadIdx.x] = g[j].bits;
    }
    const bool cut = (start & ((1u << Tc) - 1)) != 0;          // nothing passes the lane's steps, whatever their other decays are
    float A_before[V], H_before[V], A_after[V], R_after[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        A[v] = cut ? 0.0f : decayed(A[v]);
        A_before[v] = A_after[v] = 1.0f;
        H_before[v] = R_after[v] = 0.0f;
        if constexpr (V == 2) {
            const float oA = __shfl_xor(A[v], 32), oH = __shfl_xor(H[v], 32), oR = __shfl_xor(R[v], 32);
            if (group == 1) { A_before[v] = oA; H_before[v] = oH; H[v] = follow(A[v], oH, H[v]); }
            else { A_after[v] = oA; R_after[v] = oR; R[v] = follow(A[v], oR, R[v]); }
            A[v] = both(A[v], oA);
        }
        if (group == V - 1) { A_s[wave][cl + v] = A[v]; H_s[wave][cl + v] = H[v]; }
        if (group == 0) R_s[wave][cl + v] = R[v];
    }
    lds_barrier();
    if (wave == 0) {
        const int ch = at.c0 + lane;
        const bool mine = ch < p.C;
        float h = mine && p.T > 0 ? p.states[((int64_t)at.b * p.kept + unit) * p.C + ch] : 0.0f;
        float D = 0.0f, Aw = 1.0f, Rw = 0.0f;
#pragma unroll 1
        for (int w = NW - 1; w >= 0; --w) { Rw = follow(A_s[w][lane], Rw, R_s[w][lane]); Aw = both(Aw, A_s[w][lane]); }
        if constexpr (CHAIN) {
            const int64_t stride = (int64_t)p.sequences * kChannels;
            Word *own = p.words + (int64_t)at.seq * kChannels;
            if (at.unit > 0) {
                if (mine) publish(own + at.unit * stride + lane, Aw, Rw);
                D = look_back<1>(own, at.unit - 1, stride, mine, held_s);
            } else if (mine) {
                D = p.grad_h_last[(int64_t)at.b * p.C + ch];
            }
            if (mine) publish(own + at.unit * stride + lane, 0.0f, follow(Aw, D, Rw));
        } else if (mine && p.grad_h_last) {
            D = p.grad_h_last[(int64_t)at.b * p.C + ch];
        }
#pragma unroll 1
        for (int w = 0; w < NW; ++w) {
            carry_s[w][lane] = h;
            h = follow(A_s[w][lane], h, H_s[w][lane]);
        }
#pragma unroll 1
        for (int w = NW - 1; w >= 0; --w) {
            after_s[w][lane] = D;
            D = follow(A_s[w][lane], D, R_s[w][lane]);
        }
        if (mine && p.grad_h_first && unit == 0) p.grad_h_first[(int64_t)at.b * p.C + ch] = D;
    }
    lds_barrier();
    float sum[V], D[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        sum[v] = 0.0f;
        D[v] = follow(A_after[v], after_s[wave][cl + v], R_after[v]);
        float h = follow(A_before[v], carry_s[wave][cl + v], H_before[v]);
#pragma unroll
        for (int j = 0; j < Tc; ++j) {
            h = unless_start(h, start, j);
            q[j][v].q = h - q[j][v].q;
            h = fmaf(q[j][v].a, h, q[j][v].u);
        }
    }
    const int64_t last = row0 + Tc - 1;                        // (of group 0)
    Strip<E, PAIRS> sgx(p.grad_x, p.ld_gx, last, at.c0, cl, down), sgr(p.grad_r, p.ld_gr, last, at.c0, cl, down),
        sgi(p.grad_i, p.ld_gi, last, at.c0, cl, down);
    auto put = [&](auto whole) {                               // whole: every step exists and counts, and none starts a sequence
        if constexpr (CHAIN) g[Tc - 1].bits = grad_s[Tc - 1][threadIdx.x];
#pragma unroll
        for (int j = Tc - 1; j >= 0; --j) {
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (CHAIN)
                if (j > 0) g[j - 1].bits = grad_s[j - 1][threadIdx.x];
            Row<E, PAIRS> gx, gr, gi;
            float gv[V], dx[V], dr[V], di[V];
            g[j].get(gv);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const StepBack &k = q[j][v];
                const float dh = gv[v] + D[v];
                dx[v] = dh * k.m;
                di[v] = dh * k.n;
                D[v] = whole ? k.a * dh : unless_start(k.a * dh, start, j);
                const Sigmoid sr = sigmoid_of_odds(k.odds);
                const float part = whole ? sr.s * (D[v] * k.q) : unless_start(sr.s * (D[v] * k.q), start | ~filled, j);
                dr[v] = -rate[v] * (sr.c * part);
                sum[v] -= part;
            }
            gx.set(dx);
            gr.set(dr);
            gi.set(di);
            if (!whole) {                                      // padding: products with 0 would let an infinity or NaN that passes it show
                const uint32_t m = all_of(filled, j);
                gx.keep(m);
                gr.keep(m);
                gi.keep(m);
            }
            if (left > 0 && (whole || (exist >> j & 1))) {
                sgx.store(gx, left);
                sgr.store(gr, left);
                sgi.store(gi, left);
            }
            sgx.base -= sgx.step;
            sgr.base -= sgr.step;
            sgi.base -= sgi.step;
        }
    };
    if (steps.filled == (unsigned)kAll && !steps.start) put(std::true_type{});
    else put(std::false_type{});
    // the unit's part of the sum for lam: groups, then waves, in order
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if constexpr (V == 2) sum[v] += __shfl_xor(sum[v], 32);
        if (group == 0) H_s[wave][cl + v] = sum[v];
    }
    lds_barrier();
    for (int k = threadIdx.x; k < kChannels; k += NW * kWave) {
        if (at.c0 + k >= p.C) continue;
        float total = 0.0f;
        for (int w = 0; w < NW; ++w) total += H_s[w][k];
        p.lam_part[((int64_t)at.b * p.units + unit) * p.C + at.c0 + k] = total;
    }
}

// grad_lam[c] = decay sigmoid(lam[c]) * sum of the units' parts: 64 runs of each of 16 channels side by side, then together,
// in order.
__global__ __launch_bounds__(1024) void scan_lam_kernel(ScanArgs p, int64_t parts)
{
    __shared__ float run[64][16 + 1];
    const int k = threadIdx.x % 16, part = threadIdx.x / 16, c = blockIdx.x * 16 + k;
    float sum = 0.0f;
    if (c < p.C) {
#pragma unroll 4
        for (int64_t at = part; at < parts; at += 64) sum += p.lam_part[at * p.C + c];
    }
    run[part][k] = sum;
    __syncthreads();
    if (part != 0 || c >= p.C) return;
    for (int w = 1; w < 64; ++w) sum += run[w][k];
    p.grad_lam[c] = sum * p.decay * sigmoid2(p.lam[c]).s;
}

struct StepArgs {
    int n, C, slots;
    int rows_step;                     // rows that are under way at a time
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

// A single step.  A thread takes V channels, four where rows allow 16 bytes of the fp32 table at a time, else one, and every rows_step-th row:
// the rate of a channel, a third of a step's instructions, is formed once for them.  Bound by bytes where there are many rows and by
// the launch where there are few: 2048 x 4096 bf16 takes 22 us, 6.0 TB/s (33 us with an entry a thread), 777 x 2048 bf16 7 us, 24 x 64
// fp32 2.5 us.
template <typename E, int V>
__global__ __launch_bounds__(256) void step_kernel(StepArgs p)
{
    typedef E Vec __attribute__((ext_vector_type(V)));
    typedef float Floats __attribute__((ext_vector_type(V)));
    const unsigned id = blockIdx.x * 256 + threadIdx.x, per = (unsigned)p.C / V, first = id / per;
    if (first >= (unsigned)p.rows_step) return;
    const int c = (int)(id - first * per) * V;
    float rate2[V];
#pragma unroll
    for (int v = 0; v < V; ++v) rate2[v] = -kLog2e * rate_of(p.lam[c + v], p.decay);
    for (int64_t row = first; row < p.n; row += p.rows_step) {
        const int64_t at = (int64_t)(p.slot ? min(max(p.slot[row], 0), p.slots - 1) : (int)row) * p.C + c;
        const Vec x = *reinterpret_cast<const Vec *>(static_cast<const E *>(p.x) + row * p.ld_x + c);
        const Vec r = *reinterpret_cast<const Vec *>(static_cast<const E *>(p.r) + row * p.ld_r + c);
        const Vec i = *reinterpret_cast<const Vec *>(static_cast<const E *>(p.i) + row * p.ld_i + c);
        const Floats before = *reinterpret_cast<const Floats *>(p.h_in + at);
        const bool start = p.reset && p.reset[row];
        Floats h;
        Vec y;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Step s = step_of(to_f32((E)x[v]), start ? 0.0f : to_f32((E)r[v]), to_f32((E)i[v]), rate2[v], start ? -200.0f : 0.0f);
            h[v] = start ? s.u : fmaf(s.a, before[v], s.u);
            y[v] = from_f32<E>(h[v]);
        }
        *reinterpret_cast<Floats *>(p.h_out + at) = h;
        *reinterpret_cast<Vec *>(static_cast<E *>(p.y) + row * p.ld_y + c) = y;
    }
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
    const int V = 4 / element_bytes(dtype), steps = V * kSteps, steps_back = 16;
    ScanPlan s{};
    s.waves = waves_for(T, steps, kMostWaves);
    s.waves_back = waves_for(T, steps_back, T <= kMostWaves * steps_back ? kMostWaves : kMostWavesBack);
    auto units = [&](int span) { return T > 0 ? (T + span - 1) / span : 1; };
    s.units = units(s.waves * steps);
    s.units_back = units(s.waves_back * steps_back);
    s.tiles = (C + kChannels - 1) / kChannels;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    s.states = take((size_t)B * s.units_back * C * sizeof(float));
    s.aside = take((size_t)B * C * sizeof(float));
    s.n_words = s.units_back > 1 ? (int64_t)s.units_back * B * s.tiles * kChannels : 0;       // never fewer units than forward
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

// A lane's offset behind its wave's first row is held in 32 bits (Strip::lane): sixteen rows of 16-bit elements down (fp32: none), and its
// channel, less than kChannels to the right.
constexpr int64_t kWidestRow = ((int64_t)1 << 27) - kChannels;
static_assert((kSteps * kWidestRow + kChannels) * 2 <= ((int64_t)1 << 32), "");
bool rows_ok(int C, std::initializer_list<int64_t> strides)
{
    for (int64_t ld : strides)
        if (ld < C || ld > kWidestRow) return false;
    return true;
}

unsigned blocks_of(int64_t n) { return (unsigned)((n + 255) / 256); }

// Rows can be read four bytes at a time.
bool rows_of_pairs(int dtype, int C, std::initializer_list<const void *> pointers, std::initializer_list<int64_t> strides)
{
    const int V = 4 / element_bytes(dtype);
    bool ok = C % V == 0;
    for (const void *p : pointers) ok = ok && aligned_to(p, 4);
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
    default: return f(std::integral_constant<int, 8>{});
    }
}

template <bool BACK, typename E, bool PAIRS, int NW, bool CHAIN>
int launch_scan(const ScanArgs &p, hipStream_t stream)
{
    const dim3 grid((unsigned)(p.units * p.sequences)), block(NW * kWave);
    if constexpr (BACK) hipLaunchKernelGGL((scan_grad_kernel<E, PAIRS, NW, CHAIN>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((scan_kernel<E, PAIRS, NW, CHAIN>), grid, block, 0, stream, p);
    return launched(BACK ? "linear scan gradient" : "linear scan");
}

// One workgroup per unit; with more than one unit in a sequence they hand the state on.
template <bool BACK>
int run_scan(int dtype, ScanArgs p, const ScanPlan &s, char *workspace, bool pairs, hipStream_t stream)
{
    p.tiles = s.tiles;
    if ((int64_t)p.B * s.tiles * (BACK ? s.units_back : s.units) >= ((int64_t)1 << 31)) return MARL_ERR_BAD_DIM;
    p.sequences = p.B * s.tiles;
    p.units = BACK ? s.units_back : s.units;
    p.states = reinterpret_cast<float *>(workspace + s.states);
    p.kept = s.units_back;
    p.keep_log = __builtin_ctz(s.waves_back * 16);
    p.lam_part = reinterpret_cast<float *>(workspace + s.lam_part);
    p.words = reinterpret_cast<Word *>(workspace + s.words);
    p.ticket = reinterpret_cast<unsigned *>(workspace + s.ticket);
    if (p.units > 1) {
        float *aside = reinterpret_cast<float *>(workspace + s.aside);
        const int64_t n_states = (int64_t)p.B * p.C, n_words = (int64_t)p.units * p.sequences * kChannels;
        hipLaunchKernelGGL(scan_begin_kernel, dim3(blocks_of(n_words > n_states ? n_words : n_states)), dim3(256), 0, stream, p.words, n_words, p.ticket,
                           BACK ? p.grad_h_last : p.h_first, aside, n_states);
        (BACK ? p.grad_h_last : p.h_first) = aside;
        constexpr int kMost = BACK ? kMostWavesBack : kMostWaves;
        return with_dtype(dtype, [&](auto e) {
            return pairs ? launch_scan<BACK, decltype(e), true, kMost, true>(p, stream) : launch_scan<BACK, decltype(e), false, kMost, true>(p, stream);
        });
    }
    return with_dtype(dtype, [&](auto e) {
        return with_waves(BACK ? s.waves_back : s.waves, [&](auto waves) {
            return pairs ? launch_scan<BACK, decltype(e), true, decltype(waves)::value, false>(p, stream)
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
    if (!rows_ok(C, {ld_x, ld_r, ld_i, ld_y})) return MARL_ERR_BAD_DIM;
    if (T > 0 && (y == x || y == r || y == i)) return MARL_ERR_BAD_ARG;
    ScanArgs p{};
    p.B = B; p.T = T; p.C = C;
    p.x = x; p.r = r; p.i = i; p.ld_x = ld_x; p.ld_r = ld_r; p.ld_i = ld_i;
    p.lam = lam; p.decay = decay; p.reset = reset; p.filled = filled; p.h_first = h_first;
    p.y = y; p.ld_y = ld_y; p.h_last = h_last;
    const bool pairs = rows_of_pairs(dtype, C, {x, r, i, y}, {ld_x, ld_r, ld_i, ld_y});
    return run_scan<false>(dtype, p, scan_plan(dtype, B, T, C), static_cast<char *>(workspace), pairs, static_cast<hipStream_t>(hip_stream));
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
    if (!rows_ok(C, {ld_x, ld_r, ld_i, ld_gy, ld_gx, ld_gr, ld_gi})) return MARL_ERR_BAD_DIM;
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
        const bool pairs = rows_of_pairs(dtype, C, {x, r, i, grad_y, grad_x, grad_r, grad_i}, {ld_x, ld_r, ld_i, ld_gy, ld_gx, ld_gr, ld_gi});
        const int status = run_scan<true>(dtype, p, s, static_cast<char *>(workspace), pairs, stream);
        if (status) return status;
        p.lam_part = reinterpret_cast<float *>(static_cast<char *>(workspace) + s.lam_part);
    }
    hipLaunchKernelGGL(scan_lam_kernel, dim3((unsigned)((C + 15) / 16)), dim3(1024), 0, stream, p, (int64_t)B * s.units_back);
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
    StepArgs p{n, C, slots, 0, x, r, i, ld_x, ld_r, ld_i, lam, decay, slot, reset, h_in, h_out, y, ld_y};
    const size_t four = 4 * (size_t)element_bytes(dtype);
    bool fours = C % 4 == 0 && aligned_to(h_in, 16) && aligned_to(h_out, 16);
    for (const void *v : {x, r, i, static_cast<const void *>(y)}) fours = fours && aligned_to(v, four);
    for (int64_t ld : {ld_x, ld_r, ld_i, ld_y}) fours = fours && ld % 4 == 0;
    const int per = fours ? C / 4 : C, most = 256 * 2048;              // threads that the chip holds at a time
    p.rows_step = std::min(n, std::max(1, most / per));
    const dim3 grid(blocks_of((int64_t)p.rows_step * per));
    return with_dtype(dtype, [&](auto e) {
        if (fours) hipLaunchKernelGGL((step_kernel<decltype(e), 4>), grid, dim3(256), 0, static_cast<hipStream_t>(hip_stream), p);
        else hipLaunchKernelGGL((step_kernel<decltype(e), 1>), grid, dim3(256), 0, static_cast<hipStream_t>(hip_stream), p);
        return launched("linear step");
    });
}

}  // extern "C"
