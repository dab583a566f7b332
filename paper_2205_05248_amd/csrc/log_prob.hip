// Log probability of given tokens, entropy and most likely alternatives of rows of logits, and the logits' gradient.
// One pass with a running maximum m, sum s = sum e^(z-m) and moment w = sum e^(z-m) (z-m), from which log_sum = m + log s and
// entropy = log s - w / s.  Forward and backward are bound by the bytes of the logits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <limits>

#include "device_math.h"
#include "operator_types.h"

namespace marl {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTop = 64;
constexpr float kInf = __builtin_inff();

struct LogProbArgs {
    int R, V, K;
    const void *logits;
    int64_t ld;
    const int32_t *token;
    const uint8_t *avail;
    int64_t ld_avail;
    float scale;
    float lowest;                      // what is below it has a z of -infinity, and no probability
    float *logp, *entropy, *log_sum;
    int32_t *top_id;
    float *top_logp;
    // gradient
    const float *in_log_sum, *in_entropy, *grad_logp, *grad_entropy;
    void *grad_logits;
    int64_t ld_grad;
    // long rows in parts
    int parts, per;                    // parts of a row, chunks of a part
    float *stats;                      // [R, parts, 4]
    unsigned long long *keys;          // [R, parts, K]
};

// Running statistics of a set of z; m = -inf is the empty set.
struct Stats {
    float m, s, w;
};

// Distances end at kFar, where e^ is 0 in fp32: the distance of a type's lowest value would make the product 0 * infinity.
constexpr float kFar = -200.0f;

__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(kLog2e * v); }

// w of a set moved from maximum m to M >= m:  sum e^(z-M) (z-M) = e^(m-M) (w + (m-M) s).  NaN in m stays.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ Stats move_to(Stats a, float M)
{
    const float d = fmaxf(a.m - M, kFar), e = exp_of(d);
    return {M, a.s * e, e * fmaf(d, a.s, a.w)};
}
__device__ __forceinline__ Stats join(Stats a, Stats b)
{
    const float M = max_nan(a.m, b.m);
    a = move_to(a, M);
    b = move_to(b, M);
    return {M, a.s + b.s, a.w + b.w};
}
template <int LANES>
__device__ __forceinline__ Stats join_lanes(Stats st)
{
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) st = join(st, {__shfl_xor(st.m, d), __shfl_xor(st.s, d), __shfl_xor(st.w, d)});
    return st;
}

// scale * logit, rounded on its own wherever it is used: the distance of the likeliest entry is exactly 0 (fused with the subtraction it
// would be what the maximum's rounding left out), so that a lone entry has log probability 0 and none comes out above it.
__device__ __forceinline__ float rounded(float scale, float logit)
{
#pragma clang fp contract(off)
    return scale * logit;
}

// Takes in N logits, -inf where there is none.  A row's maximum settles after a few calls.
template <int N>
__device__ __forceinline__ void take(Stats &st, const float (&l)[N], float scale)
{
    float top = l[0];
#pragma unroll
    for (int k = 1; k < N; ++k) top = max_nan(top, l[k]);
    const float M = max_nan(st.m, top == -kInf ? -kInf : rounded(scale, top));
    if (!(M == st.m)) st = move_to(st, M);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        // nothing there: the distance ends at -1e30, whose exponential is 0.  NaN too, but then M is NaN, which is what counts.
        const float d = fmaxf(rounded(scale, l[k]) - M, -1e30f), e = exp_of(d);
        st.s += e;
        st.w = fmaf(e, d, st.w);
    }
}

// The value that a lane D away holds; from D = 4 on where lanes of the same quad (eight, for D = 8) hold the same.
template <int D>
__device__ __forceinline__ float across(float v)
{
    constexpr int kControl = D == 1 ? 0xb1 : D == 2 ? 0x4e : D == 4 ? 0x141 : 0x140;       // within quads; mirrored eights; mirrored sixteens
    if constexpr (D <= 8) return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kControl, 0xf, 0xf, true));
    else return __shfl_xor(v, D);
}
template <int LANES, int D = 1, class F>
__device__ __forceinline__ float all_lanes(float v, F &&join)
{
    if constexpr (D < LANES) return all_lanes<LANES, 2 * D>(join(v, across<D>(v)), join);
    else return v;
}

// Statistics of a row that LANES lanes hold whole: the maximum first, then the sums, nothing is moved.  (Running statistics, joined lane by
// lane, were 290 instructions of a wave for 8 rows of 40, and instructions bound it.)
template <int LANES, int N>
__device__ __forceinline__ Stats stats_of(const float (&l)[N], float scale)
{
    float top = l[0];
#pragma unroll
    for (int k = 1; k < N; ++k) top = max_nan(top, l[k]);
    top = all_lanes<LANES>(top, [](float a, float b) { return max_nan(a, b); });
    Stats st{top == -kInf ? -kInf : rounded(scale, top), 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float d = fmaxf(rounded(scale, l[k]) - st.m, -1e30f), e = exp_of(d);         // as in take
        st.s += e;
        st.w = fmaf(e, d, st.w);
    }
    st.s = all_lanes<LANES>(st.s, [](float a, float b) { return a + b; });
    st.w = all_lanes<LANES>(st.w, [](float a, float b) { return a + b; });
    return st;
}

// What a row's statistics and its token give.  A maximum of NaN or +infinity makes everything NaN.
__device__ __forceinline__ void put_row(const LogProbArgs &p, int64_t row, Stats st, bool available, float logit, int token)
{
    const bool none = st.m == -kInf, bad = !(st.m < kInf);
    const float nan = __builtin_nanf(""), log_s = logf(st.s);
    if (p.log_sum) p.log_sum[row] = bad ? nan : none ? -kInf : st.m + log_s;
    if (p.entropy) p.entropy[row] = bad ? nan : none ? 0.0f : log_s - st.w / st.s;
    if (p.logp) {
        float lp = 0.0f;
        if (token >= 0 && token < p.V) lp = bad ? nan : none ? 0.0f : !available || logit < p.lowest ? -kInf : (rounded(p.scale, logit) - st.m) - log_s;
        else if (bad) lp = nan;
        p.logp[row] = lp;
    }
}

template <typename E>
__device__ __forceinline__ void finish_row(const LogProbArgs &p, int64_t row, Stats st)
{
    const int token = p.logp ? p.token[row] : -1;
    const bool in = token >= 0 && token < p.V;
    put_row(p, row, st, in && (!p.avail || p.avail[row * p.ld_avail + token]), in ? to_f32(static_cast<const E *>(p.logits)[row * p.ld + token]) : 0.0f, token);
}

// ---------------------------------------------------------------------------------- the K largest of what a wave holds
// Keys order values, and equal values by lower index; 0 is nothing.
typedef unsigned long long Key;

__device__ __forceinline__ unsigned order_of(float v)
{
    const unsigned u = __float_as_uint(v + 0.0f);                      // -0 is 0
    return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(Key key)
{
    const unsigned u = (unsigned)(key >> 32);
    return __uint_as_float(u ^ (u >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ Key key_of(unsigned order, unsigned index) { return order ? (Key)order << 32 | (unsigned)~index : 0; }
__device__ __forceinline__ unsigned index_of(Key key) { return ~(unsigned)key; }

__device__ __forceinline__ Key lane_key(Key key, int lane)
{
    return (Key)(unsigned)__builtin_amdgcn_readlane((int)(key >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)key, lane);
}

__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// out[0 .. K) = the K largest of 64 N entries in descending order, 0 behind the last.  The K-th largest of the lanes' own
// largest bounds the K-th largest of all from below, and only K lanes have anything that reaches it: what reaches it goes to
// `kept` (room for K N keys) and is ordered by counting.  For K = 20 of random values 24 of 2048 reach it.
// RISING: a lane's indexes rise with j, so that of equal values it meets the first one first.
template <int N, bool RISING, class OrderAt, class IndexAt>
__device__ __forceinline__ void wave_top(OrderAt order, IndexAt index, int K, Key *kept, Key *out)
{
    const int lane = threadIdx.x % kWave;
    Key mine = 0;
    if constexpr (RISING) {
        unsigned best = 0, at = 0;
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (order(j) > best) { best = order(j); at = index(j); }
        mine = key_of(best, at);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const Key key = key_of(order(j), index(j));
            mine = key > mine ? key : mine;
        }
    }
    int above = 0;
    for (int l = 0; l < kWave; ++l) above += lane_key(mine, l) > mine;
    const unsigned long long at_k = __ballot(above == K - 1 && mine);
    const Key least = at_k ? lane_key(mine, __ffsll((long long)at_k) - 1) : 1;
    int n = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const Key key = key_of(order(j), index(j));
        const unsigned long long pass = __ballot(key >= least);
        if (pass) {
            if (key >= least) kept[n + __popcll(pass & ((1ull << lane) - 1))] = key;
            n += __popcll(pass);
        }
    }
    wave_sync();
    for (int c = lane; c < n; c += kWave) {
        const Key key = kept[c];
        int rank = 0;
        for (int q = 0; q < n; ++q) rank += kept[q] > key;
        if (rank < K) out[rank] = key;
    }
    for (int c = n + lane; c < K; c += kWave) out[c] = 0;
    wave_sync();
}

__device__ __forceinline__ void put_top(const LogProbArgs &p, int64_t row, int k, Key key, Stats st, float log_s)
{
    p.top_id[row * p.K + k] = key ? (int)index_of(key) : -1;
    p.top_logp[row * p.K + k] = key ? (rounded(p.scale, value_of(key)) - st.m) - log_s : -kInf;
}

// ---------------------------------------------------------------------------------- reading
// 16 bytes of a row at any element alignment, and as many mask bytes.
template <typename E>
struct Piece {
    static constexpr int V = 16 / (int)sizeof(E);
    typedef E Vec __attribute__((ext_vector_type(V)));
    typedef Vec Loose __attribute__((aligned(sizeof(E))));
    typedef uint8_t Bytes __attribute__((ext_vector_type(V)));
    typedef Bytes LooseBytes __attribute__((aligned(1)));
};

// How many entries a row begins behind a line of 128 bytes.  Pieces are counted from there, so that a wave reads and writes whole
// lines: 8191 rows of 50021 in fp16 took 194 us forward and 364 us backward from where they begin, 165 and 364 us from a multiple of 16
// bytes on, and take 160 and 334 us.
template <typename E>
__device__ __forceinline__ int skew_of(const E *l) { return (int)((reinterpret_cast<uintptr_t>(l) & 127) / sizeof(E)); }

// Entries j .. j + V of a row as fp32, -inf where masked, before entry `first` or behind the end.
template <typename E>
__device__ __forceinline__ void read_piece(const E *l, const uint8_t *av, int j, int first, int V, float *to)
{
    typedef Piece<E> P;
    if (j >= first && j + P::V <= V) {
        const typename P::Vec v = *reinterpret_cast<const typename P::Loose *>(l + j);
#pragma unroll
        for (int k = 0; k < P::V; ++k) to[k] = to_f32(v[k]);
        if (av) {
            const typename P::Bytes m = *reinterpret_cast<const typename P::LooseBytes *>(av + j);
#pragma unroll
            for (int k = 0; k < P::V; ++k) to[k] = m[k] ? to[k] : -kInf;
        }
    } else {
#pragma unroll
        for (int k = 0; k < P::V; ++k) to[k] = j + k >= first && j + k < V && (!av || av[j + k]) ? to_f32(l[j + k]) : -kInf;
    }
}

// ---------------------------------------------------------------------------------- long rows
constexpr int kHeld = 32;                              // logits of a lane at a time
constexpr int kChunk = kThreads * kHeld;               // of a workgroup

// A workgroup takes `per` chunks of a row; with one part per row it finishes the row, otherwise join_kernel does.  With
// alternatives a part is one chunk, which stays in registers for wave_top.  8191 x 50021 fp16: 160 us, 5.1 TB/s, 11 instructions a logit.
// 16 x 131072 bf16 with twenty alternatives: 13 us, and 6 us for the join; 256 workgroups of one chunk each, so what it costs is
// one chunk's chain of loads, ballots and counts.
template <typename E, bool TOP>
__global__ __launch_bounds__(kThreads) void long_rows_kernel(LogProbArgs p)
{
    constexpr int V = Piece<E>::V;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ Stats part[kThreads / kWave];
    const int64_t row = blockIdx.x / p.parts;
    const int piece = blockIdx.x % p.parts;
    const E *l = static_cast<const E *>(p.logits) + row * p.ld;
    const uint8_t *av = p.avail ? p.avail + row * p.ld_avail : nullptr;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int skew = TOP ? 0 : skew_of(l), n = p.V + skew;             // entry j of the row is skew + j
    l -= skew;
    if (av) av -= skew;
    const int64_t begin = (int64_t)piece * p.per * kChunk, end = piece + 1 < p.parts ? begin + (int64_t)p.per * kChunk : n;
    Stats st{-kInf, 0.0f, 0.0f};
    float held[kHeld];
    int64_t base = begin;
    for (; TOP ? base < end : base + kChunk <= end; base += kChunk) {
#pragma unroll
        for (int q = 0; q < kHeld / V; ++q) read_piece<E>(l, av, (int)base + (q * kThreads + (int)threadIdx.x) * V, skew, n, held + q * V);
        take(st, held, p.scale);
    }
    if constexpr (!TOP) {                                              // what is left: a piece at a time, and no more than there are
        for (; base + wave * (kWave * V) < end; base += kThreads * V) {
            float some[V];
            read_piece<E>(l, av, (int)base + (int)threadIdx.x * V, skew, n, some);
            take(st, some, p.scale);
        }
    }
    st = join_lanes<kWave>(st);
    if (lane == 0) part[wave] = st;
    if constexpr (TOP) {
        const int K = p.K;
        Key *lists = reinterpret_cast<Key *>(lds), *kept = lists + (kThreads / kWave) * K + (size_t)wave * K * kHeld;
        wave_top<kHeld, true>([&](int j) { return held[j] < p.lowest ? 0u : order_of(held[j]); },
                        [&](int j) { return (unsigned)((int)begin + (j / V * kThreads + (int)threadIdx.x) * V + j % V); }, K, kept, lists + wave * K);
    }
    __syncthreads();
    if (wave != 0) return;
    st = part[0];
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) st = join(st, part[w]);
    if constexpr (TOP) {
        const int K = p.K;
        Key *lists = reinterpret_cast<Key *>(lds), *kept = lists + (kThreads / kWave) * K;
        Key own[kThreads / kWave];
#pragma unroll
        for (int w = 0; w < kThreads / kWave; ++w) own[w] = lane < K ? lists[w * K + lane] : 0;
        wave_sync();
        wave_top<kThreads / kWave, false>([&](int j) { return (unsigned)(own[j] >> 32); }, [&](int j) { return index_of(own[j]); }, K, kept, lists);
        if (lane < K) {
            if (p.parts > 1) p.keys[((int64_t)row * p.parts + piece) * K + lane] = lists[lane];
            else put_top(p, row, lane, lists[lane], st, logf(st.s));
        }
    }
    if (lane == 0) {
        if (p.parts > 1) {
            float *to = p.stats + ((int64_t)row * p.parts + piece) * 4;
            to[0] = st.m; to[1] = st.s; to[2] = st.w;
        } else {
            finish_row<E>(p, row, st);
        }
    }
}

// A wave per row joins its parts.
template <typename E>
__global__ __launch_bounds__(kWave) void join_kernel(LogProbArgs p)
{
    constexpr int N = 8;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x, K = p.K;
    Stats st{-kInf, 0.0f, 0.0f};
    for (int k = lane; k < p.parts; k += kWave) {
        const float *from = p.stats + (row * p.parts + k) * 4;
        st = join(st, {from[0], from[1], from[2]});
    }
    st = join_lanes<kWave>(st);
    if (K > 0) {
        Key *out = reinterpret_cast<Key *>(lds), *kept = out + K;
        const Key *from = p.keys + row * p.parts * K;
        const int64_t n = (int64_t)p.parts * K;
        bool first = true;
        for (int64_t base = 0; base < n; first = false) {              // the K best so far, and as many more as there is room for
            Key own[N];
            own[0] = first ? 0 : lane < K ? out[lane] : 0;
#pragma unroll
            for (int j = 1; j < N; ++j) {
                const int64_t k = base + (int64_t)(j - 1) * kWave + lane;
                own[j] = k < n ? from[k] : 0;
            }
            base += (N - 1) * kWave;
            wave_sync();
            wave_top<N, false>([&](int j) { return (unsigned)(own[j] >> 32); }, [&](int j) { return index_of(own[j]); }, K, kept, out);
        }
        if (lane < K) put_top(p, row, lane, out[lane], st, logf(st.s));
    }
    if (lane == 0) finish_row<E>(p, row, st);
}

// ---------------------------------------------------------------------------------- short rows
// Rows that follow one another without a gap (FLAT): a wave brings its 64 / G of them to shared memory as one stretch, 16 bytes a
// lane, and the lanes of a row take their entries from there.  A row of forty alone is 32 bytes a load and lane group, and loads, not
// bytes, bound it: with a load per row 409600 x 40 fp32 with a mask took 31 us forward and 38 us backward.
// `at`, `count`: the wave's stretch of an array of `total`; returns where in `to` it begins.
template <typename T, int MOST>
__device__ __forceinline__ int bring(const T *from, int64_t total, int64_t at, int count, T *to)
{
    constexpr int V = 16 / (int)sizeof(T), kTurns = (MOST + V - 1 + kWave * V - 1) / (kWave * V);
    typedef T Vec __attribute__((ext_vector_type(V)));
    const int skew = (int)((reinterpret_cast<uintptr_t>(from + at) & 15) / sizeof(T));
    Vec v[kTurns];
#pragma unroll
    for (int q = 0; q < kTurns; ++q) {
        const int piece = (q * kWave + (int)threadIdx.x % kWave) * V;
        const int64_t j = at - skew + piece;
        if (piece >= skew + count) continue;
        if (j >= 0 && j + V <= total) {
            v[q] = *reinterpret_cast<const Vec *>(from + j);
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k) v[q][k] = j + k >= 0 && j + k < total ? from[j + k] : (T)0;
        }
    }
#pragma unroll
    for (int q = 0; q < kTurns; ++q) {
        const int piece = (q * kWave + (int)threadIdx.x % kWave) * V;
        if (piece < skew + count) *reinterpret_cast<Vec *>(to + piece) = v[q];
    }
    return skew;
}
// And back, the stretch alone; `from` begins at the skew of `to + at`.
template <typename T, int MOST>
__device__ __forceinline__ void bring_back(T *to, int64_t at, int count, int skew, const T *from)
{
    constexpr int V = 16 / (int)sizeof(T), kTurns = (MOST + V - 1 + kWave * V - 1) / (kWave * V);
    typedef T Vec __attribute__((ext_vector_type(V)));
#pragma unroll
    for (int q = 0; q < kTurns; ++q) {
        const int piece = (q * kWave + (int)threadIdx.x % kWave) * V;
        if (piece >= skew + count) continue;
        T *out = to + at - skew + piece;
        if (piece >= skew && piece + V <= skew + count) {
            *reinterpret_cast<Vec *>(out) = *reinterpret_cast<const Vec *>(from + piece);
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (piece + k >= skew && piece + k < skew + count) out[k] = from[piece + k];
        }
    }
}
// Room of a wave, in entries: a stretch, what lies before it and the end of its last piece.
template <typename T, int MOST> constexpr int kStretch = (MOST + 2 * (16 / (int)sizeof(T)) - 1) / (16 / (int)sizeof(T)) * (16 / (int)sizeof(T));

// The wave's rows through shared memory: entry j G + sub of the lane's row, -inf where masked or not there.
template <typename E, int G, int N>
struct FlatRows {
    static constexpr int kMost = kWave * N;
    E entries[kStretch<E, kMost>];
    uint8_t mask[kStretch<uint8_t, kMost>];
    // token: of the lane's row, or -1; its logit and whether it is available are left in `taken`
    struct Taken { float logit; bool available; };
    __device__ __forceinline__ Taken read(const LogProbArgs &p, int64_t first, int64_t row, bool there, int token, float (&held)[N])
    {
        const int sub = threadIdx.x % G, rows = (int)min((int64_t)(kWave / G), p.R - first);
        const int64_t at = first * p.V, total = (int64_t)p.R * p.V;
        const bool own = p.avail && p.ld_avail != 0;
        const int skew = bring<E, kMost>(static_cast<const E *>(p.logits), total, at, rows * p.V, entries);
        const int skew_m = own ? bring<uint8_t, kMost>(p.avail, total, at, rows * p.V, mask) : 0;
        wave_sync();
        const int in = (int)(row - first) * p.V;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int k = j * G + sub;
            const bool is = there && k < p.V && (!p.avail || (own ? mask[skew_m + in + k] : p.avail[k]));
            held[j] = is ? to_f32(entries[skew + in + k]) : -kInf;
        }
        const bool in_row = there && token >= 0 && token < p.V;
        const Taken taken{in_row ? to_f32(entries[skew + in + token]) : -kInf,
                          in_row && (!p.avail || (own ? mask[skew_m + in + token] : p.avail[token]))};
        wave_sync();
        return taken;
    }
};

// G lanes hold a row of at most G N logits; a wave takes 64 / G rows.  409600 x 40 fp32 with a mask: 24 us forward (3.5 TB/s, its
// instructions bound it), 29 us backward (5 TB/s).  20000 x 1000 fp32: 46 us both ways; bf16 72 us, for a lane reads an entry at a time.
// Alternatives of rows up to 256 are found by a pass each: 20000 x 256 fp32 takes 7 us without, 12 with five, 58 with fifty.
template <typename E, int G, int N, bool FLAT>
__global__ __launch_bounds__(kThreads) void short_rows_kernel(LogProbArgs p)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, sub = lane % G;
    const int64_t row = ((int64_t)blockIdx.x * (kThreads / kWave) + wave) * (kWave / G) + lane / G;
    const bool there = row < p.R;
    const E *l = static_cast<const E *>(p.logits) + (there ? row : 0) * p.ld;
    const uint8_t *av = p.avail ? p.avail + (there ? row : 0) * p.ld_avail : nullptr;
    float held[N];
    const int token = there && p.logp ? p.token[row] : -1;
    typename FlatRows<E, G, N>::Taken taken;
    if constexpr (FLAT) {
        __shared__ __attribute__((aligned(16))) FlatRows<E, G, N> rows[kThreads / kWave];
        const int64_t first = ((int64_t)blockIdx.x * (kThreads / kWave) + wave) * (kWave / G);
        if (first >= p.R) return;                                      // the whole wave
        taken = rows[wave].read(p, first, row, there, token, held);
    } else {
        const bool in = token >= 0 && token < p.V;
        taken = {in ? to_f32(l[token]) : -kInf, in && (!av || av[token])};
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int k = j * G + sub;
            held[j] = there && k < p.V && (!av || av[k]) ? to_f32(l[k]) : -kInf;
        }
    }
    const Stats st = stats_of<G>(held, p.scale);
    if (there && sub == 0) put_row(p, row, st, taken.available, taken.logit, token);
    if (p.K == 0) return;
    const float log_s = logf(st.s);
    if constexpr (G == kWave) {
        if (!there) return;                                            // the whole wave
        Key *out = reinterpret_cast<Key *>(lds) + (size_t)wave * p.K * (N + 1), *kept = out + p.K;
        wave_top<N, true>([&](int j) { return held[j] < p.lowest ? 0u : order_of(held[j]); }, [&](int j) { return (unsigned)(j * G + sub); }, p.K, kept, out);
        if (lane < p.K) put_top(p, row, lane, out[lane], st, log_s);
    } else {
        Key last = ~(Key)0;
        for (int k = 0; k < p.K; ++k) {                                // the largest below the last one
            Key best = 0;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const Key key = held[j] < p.lowest ? 0 : key_of(order_of(held[j]), j * G + sub);
                if (key < last && key > best) best = key;
            }
#pragma unroll
            for (int d = 1; d < G; d *= 2) {
                const Key other = (Key)(unsigned)__shfl_xor((int)(best >> 32), d) << 32 | (unsigned)__shfl_xor((int)(unsigned)best, d);
                best = other > best ? other : best;
            }
            if (there && sub == 0) put_top(p, row, k, best, st, log_s);
            last = best;
        }
    }
}

// ---------------------------------------------------------------------------------- gradient
struct RowGrad { float log_sum, ent, g_logp, g_ent; int token; };      // token: -1 without a gradient of its own; log_sum -inf: nothing there

// (every load at once, none waits for another)
__device__ __forceinline__ RowGrad row_grad(const LogProbArgs &p, int64_t row)
{
    RowGrad g;
    g.log_sum = p.in_log_sum[row];
    g.token = p.grad_logp ? p.token[row] : -1;
    g.g_logp = p.grad_logp ? p.grad_logp[row] : 0.0f;
    g.g_ent = p.grad_entropy ? p.grad_entropy[row] : 0.0f;
    g.ent = p.grad_entropy ? p.in_entropy[row] : 0.0f;
    return g;
}
// A token that is outside the row, masked or without probability has no gradient.
__device__ __forceinline__ void drop_token(RowGrad &g, bool available, float logit, float lowest)
{
    const bool has = available && !(logit < lowest);
    g.token = has ? g.token : -1;
    g.g_logp = has ? g.g_logp : 0.0f;
}
template <typename E>
__device__ __forceinline__ void look_at_token(RowGrad &g, const E *l, const uint8_t *av, int V, float lowest)
{
    const bool in = g.token >= 0 && g.token < V;
    drop_token(g, in && (!av || av[g.token]), in ? to_f32(l[g.token]) : -kInf, lowest);
}

__device__ __forceinline__ float grad_of(const RowGrad &g, float logit, bool taken, float scale, float lowest)
{
    // p as the square of its root, which the hardware exponential does not flush where p is subnormal; a log_sum of NaN stays one
    const float lp = max_nan(rounded(scale, logit) - g.log_sum, kFar), root = __builtin_amdgcn_exp2f(0.5f * kLog2e * lp);
    const float v = scale * ((taken ? g.g_logp : 0.0f) - root * (root * fmaf(g.g_ent, lp + g.ent, g.g_logp)));
    return logit < lowest || g.log_sum == -kInf ? 0.0f : v;
}

// A workgroup takes `per` chunks of a row (the whole row if it overwrites the logits: the token's is read before any is gone).
// 8191 x 50021 fp16: 334 us, 4.9 TB/s; a large copy reaches 5.25.
template <typename E>
__global__ __launch_bounds__(kThreads, 8) void long_grad_kernel(LogProbArgs p)
{
    typedef Piece<E> P;
    constexpr int V = P::V, kPieces = 4;
    const int64_t row = blockIdx.x / p.parts;
    const int piece = blockIdx.x % p.parts;
    const E *l = static_cast<const E *>(p.logits) + row * p.ld;
    const uint8_t *av = p.avail ? p.avail + row * p.ld_avail : nullptr;
    E *out = static_cast<E *>(p.grad_logits) + row * p.ld_grad;
    RowGrad g = row_grad(p, row);
    look_at_token(g, l, av, p.V, p.lowest);
    __syncthreads();
    const int skew = skew_of(l), n = p.V + skew, token = g.token + skew;           // entry j of the row is skew + j
    l -= skew;
    out -= skew;
    if (av) av -= skew;
    auto put = [&](const float *held, int j) {
        typename P::Vec v;
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = from_f32<E>(grad_of(g, held[k], j + k == token, p.scale, p.lowest));
        if (j >= skew && j + V <= n) {
            *reinterpret_cast<typename P::Loose *>(out + j) = v;
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (j + k >= skew && j + k < n) out[j + k] = v[k];
        }
    };
    constexpr int kStep = kThreads * V * kPieces;
    int64_t base = (int64_t)piece * p.per * kStep;
    const int64_t end = piece + 1 < p.parts ? base + (int64_t)p.per * kStep : n;
    for (; base + kStep <= end; base += kStep) {
        float held[kPieces][V];
#pragma unroll
        for (int q = 0; q < kPieces; ++q) read_piece<E>(l, av, (int)base + (q * kThreads + (int)threadIdx.x) * V, skew, n, held[q]);
#pragma unroll
        for (int q = 0; q < kPieces; ++q) put(held[q], (int)base + (q * kThreads + (int)threadIdx.x) * V);
    }
    for (; base + (threadIdx.x / kWave) * (kWave * V) < end; base += kThreads * V) {                       // what is left: a piece at a time
        float held[V];
        read_piece<E>(l, av, (int)base + (int)threadIdx.x * V, skew, n, held);
        put(held, (int)base + (int)threadIdx.x * V);
    }
}

template <typename E, int G, int N, bool FLAT>
__global__ __launch_bounds__(kThreads) void short_grad_kernel(LogProbArgs p)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, sub = lane % G;
    const int64_t first = ((int64_t)blockIdx.x * (kThreads / kWave) + wave) * (kWave / G), row = first + lane / G;
    if (first >= p.R) return;                                          // the whole wave
    const bool there = row < p.R;
    const int64_t own = there ? row : first;
    const E *l = static_cast<const E *>(p.logits) + own * p.ld;
    const uint8_t *av = p.avail ? p.avail + own * p.ld_avail : nullptr;
    E *out = static_cast<E *>(p.grad_logits) + own * p.ld_grad;
    RowGrad g = row_grad(p, own);
    float held[N];
    if constexpr (FLAT) {
        __shared__ __attribute__((aligned(16))) FlatRows<E, G, N> rows[kThreads / kWave];
        const auto taken = rows[wave].read(p, first, row, there, g.token, held);
        drop_token(g, taken.available, taken.logit, p.lowest);
        const int count = (int)min((int64_t)(kWave / G), p.R - first) * p.V;
        const int skew = (int)((reinterpret_cast<uintptr_t>(static_cast<E *>(p.grad_logits) + first * p.V) & 15) / sizeof(E));
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int k = j * G + sub;
            if (there && k < p.V) rows[wave].entries[skew + (int)(row - first) * p.V + k] = from_f32<E>(grad_of(g, held[j], k == g.token, p.scale, p.lowest));
        }
        wave_sync();
        bring_back<E, kWave * N>(static_cast<E *>(p.grad_logits), first * p.V, count, skew, rows[wave].entries);
    } else {
        look_at_token(g, l, av, p.V, p.lowest);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int k = j * G + sub;
            held[j] = there && k < p.V && (!av || av[k]) ? to_f32(l[k]) : -kInf;
        }
        wave_sync();                                                   // all of the row is read before any of it is overwritten
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int k = j * G + sub;
            if (there && k < p.V) out[k] = from_f32<E>(grad_of(g, held[j], k == g.token, p.scale, p.lowest));
        }
    }
}

// Rows without a gap between them, and masks too.
bool rows_are_flat(const LogProbArgs &p) { return p.ld == p.V && (!p.avail || p.ld_avail == 0 || p.ld_avail == p.V); }

// The lowest finite logit whose product with the scale, rounded to fp32, is finite.
float lowest_of(float scale)
{
    const float least = std::numeric_limits<float>::lowest();
    if (scale <= 1.0f) return least;
    float v = least / scale;                                           // within a step of it
    while (!std::isfinite(scale * v)) v = std::nextafter(v, 0.0f);
    for (float w; std::isfinite(scale * (w = std::nextafter(v, least)));) v = w;
    return v;
}

int log_prob_check(int dtype, int R, int V, const void *logits, int64_t ld, const uint8_t *avail, int64_t ld_avail, float scale)
{
    if (!known_dtype(dtype)) return MARL_ERR_BAD_DTYPE;
    if (R < 0 || V < 1 || V >= (1 << 30) || ld < V) return MARL_ERR_BAD_DIM;
    if (avail && ld_avail != 0 && ld_avail < V) return MARL_ERR_BAD_DIM;
    if (!std::isfinite(scale) || !(scale > 0.0f)) return MARL_ERR_BAD_ARG;
    return !logits && R > 0 ? MARL_ERR_NULL : MARL_OK;
}

// Rows up to this long are held by one wave or a part of it.
constexpr int kShort = 2048;

// Parts of a long row: with alternatives one per chunk; otherwise as many as fill the chip (eight workgroups on each of 256
// compute units), not less than a chunk each.
struct Cut { int parts, per; };
Cut cut_of(int R, int V, int chunk, bool one_each)
{
    const int chunks = (V + chunk - 1) / chunk;
    const int wanted = one_each ? chunks : (int)std::min<int64_t>(chunks, std::max<int64_t>(1, 2048 / std::max(R, 1)));
    const int per = (chunks + wanted - 1) / wanted;
    return {(chunks + per - 1) / per, per};
}

size_t log_prob_workspace(int R, int V, int K)
{
    if (V <= kShort) return 0;
    const Cut cut = cut_of(R, V, kChunk, K > 0);
    if (cut.parts == 1) return 0;
    const size_t n = (size_t)R * cut.parts;
    return ((n * 4 * sizeof(float) + 255) / 256 + (n * K * sizeof(Key) + 255) / 256) * 256;
}

// Shared memory beyond 64 KB (from 63 alternatives on) has to be asked for.
int make_room(void (*kernel)(LogProbArgs), size_t lds)
{
    if (lds <= 64 * 1024) return MARL_OK;
    const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    return err == hipSuccess ? MARL_OK : report_device_error(err, "hipFuncSetAttribute");
}

template <typename E>
int run_forward(LogProbArgs p, char *workspace, hipStream_t stream)
{
    if (p.V <= kShort) {
        // lanes of a row: enough to hold it, few enough that short rows share a wave
        auto go = [&](auto kernel, int G, int N) {
            const int64_t rows = (int64_t)(kThreads / kWave) * (kWave / G);
            const size_t lds = G == kWave ? (size_t)(kThreads / kWave) * p.K * (N + 1) * sizeof(Key) : 0;
            if (const int rc = make_room(kernel, lds)) return rc;
            hipLaunchKernelGGL(kernel, dim3((unsigned)((p.R + rows - 1) / rows)), dim3(kThreads), lds, stream, p);
            return launched("log prob");
        };
        if (rows_are_flat(p)) {
            if (p.V <= 16) return go(short_rows_kernel<E, 4, 4, true>, 4, 4);
            if (p.V <= 48) return go(short_rows_kernel<E, 8, 6, true>, 8, 6);
            if (p.V <= 64) return go(short_rows_kernel<E, 8, 8, true>, 8, 8);
            if (p.V <= 256) return go(short_rows_kernel<E, 16, 16, true>, 16, 16);
        }
        if (p.V <= 16) return go(short_rows_kernel<E, 4, 4, false>, 4, 4);
        if (p.V <= 64) return go(short_rows_kernel<E, 8, 8, false>, 8, 8);
        if (p.V <= 256) return go(short_rows_kernel<E, 16, 16, false>, 16, 16);
        if (p.V <= 512) return go(short_rows_kernel<E, kWave, 8, false>, kWave, 8);
        return go(short_rows_kernel<E, kWave, 32, false>, kWave, 32);
    }
    const Cut cut = cut_of(p.R, p.V, kChunk, p.K > 0);
    p.parts = cut.parts;
    p.per = cut.per;
    if ((int64_t)p.R * p.parts >= ((int64_t)1 << 31)) return MARL_ERR_BAD_DIM;
    p.stats = reinterpret_cast<float *>(workspace);
    p.keys = reinterpret_cast<Key *>(workspace + ((size_t)p.R * p.parts * 4 * sizeof(float) + 255) / 256 * 256);
    const dim3 grid((unsigned)(p.R * p.parts));
    if (p.K > 0) {
        const size_t lds = (size_t)(kThreads / kWave) * p.K * (kHeld + 1) * sizeof(Key);
        if (const int rc = make_room(long_rows_kernel<E, true>, lds)) return rc;
        hipLaunchKernelGGL((long_rows_kernel<E, true>), grid, dim3(kThreads), lds, stream, p);
    } else {
        hipLaunchKernelGGL((long_rows_kernel<E, false>), grid, dim3(kThreads), 0, stream, p);
    }
    if (p.parts > 1) hipLaunchKernelGGL(join_kernel<E>, dim3((unsigned)p.R), dim3(kWave), (size_t)p.K * 9 * sizeof(Key), stream, p);
    return launched("log prob");
}

template <typename E>
int run_backward(LogProbArgs p, hipStream_t stream)
{
    if (p.V <= kShort) {
        auto go = [&](auto kernel, int G) {
            const int64_t rows = (int64_t)(kThreads / kWave) * (kWave / G);
            hipLaunchKernelGGL(kernel, dim3((unsigned)((p.R + rows - 1) / rows)), dim3(kThreads), 0, stream, p);
            return launched("log prob gradient");
        };
        if (rows_are_flat(p) && p.ld_grad == p.V) {
            if (p.V <= 16) return go(short_grad_kernel<E, 4, 4, true>, 4);
            if (p.V <= 48) return go(short_grad_kernel<E, 8, 6, true>, 8);
            if (p.V <= 64) return go(short_grad_kernel<E, 8, 8, true>, 8);
            if (p.V <= 256) return go(short_grad_kernel<E, 16, 16, true>, 16);
        }
        if (p.V <= 16) return go(short_grad_kernel<E, 4, 4, false>, 4);
        if (p.V <= 64) return go(short_grad_kernel<E, 8, 8, false>, 8);
        if (p.V <= 256) return go(short_grad_kernel<E, 16, 16, false>, 16);
        if (p.V <= 512) return go(short_grad_kernel<E, kWave, 8, false>, kWave);
        return go(short_grad_kernel<E, kWave, 32, false>, kWave);
    }
    Cut cut = cut_of(p.R, p.V, kThreads * Piece<E>::V * 4, false);
    if (p.grad_logits == p.logits) cut = {1, cut.parts * cut.per};
    p.parts = cut.parts;
    p.per = cut.per;
    if ((int64_t)p.R * p.parts >= ((int64_t)1 << 31)) return MARL_ERR_BAD_DIM;
    hipLaunchKernelGGL((long_grad_kernel<E>), dim3((unsigned)(p.R * p.parts)), dim3(kThreads), 0, stream, p);
    return launched("log prob gradient");
}

}  // namespace
}  // namespace marl

using namespace marl;

extern "C" {

int marl_log_prob_workspace_bytes(int32_t R, int32_t V, int32_t K, size_t *bytes)
{
    if (!bytes) return MARL_ERR_NULL;
    if (R < 0 || V < 1 || V >= (1 << 30) || K < 0 || K > kMaxTop) return MARL_ERR_BAD_DIM;
    *bytes = log_prob_workspace(R, V, K);
    return MARL_OK;
}

int marl_log_prob(int32_t dtype, int32_t R, int32_t V, const void *logits, int64_t ld, const int32_t *token,
                  const uint8_t *avail, int64_t ld_avail, float scale, float *logp, float *entropy, float *log_sum,
                  int32_t K, int32_t *top_id, float *top_logp, void *workspace, size_t workspace_bytes,
                  void *hip_stream)
{
    const int rc = log_prob_check(dtype, R, V, logits, ld, avail, ld_avail, scale);
    if (rc) return rc;
    if (K < 0 || K > kMaxTop || workspace_bytes < log_prob_workspace(R, V, K)) return MARL_ERR_BAD_DIM;
    if (R == 0) return MARL_OK;
    if ((logp && !token) || (K > 0 && (!top_id || !top_logp)) || (workspace_bytes && !workspace)) return MARL_ERR_NULL;
    if (!aligned_to(workspace, 256)) return MARL_ERR_BAD_ARG;
    LogProbArgs p{};
    p.R = R; p.V = V; p.K = K;
    p.logits = logits; p.ld = ld; p.token = token; p.avail = avail; p.ld_avail = ld_avail; p.scale = scale; p.lowest = lowest_of(scale);
    p.logp = logp; p.entropy = entropy; p.log_sum = log_sum; p.top_id = top_id; p.top_logp = top_logp;
    return with_dtype(dtype, [&](auto e) { return run_forward<decltype(e)>(p, static_cast<char *>(workspace), static_cast<hipStream_t>(hip_stream)); });
}

int marl_log_prob_grad(int32_t dtype, int32_t R, int32_t V, const void *logits, int64_t ld, const int32_t *token,
                       const uint8_t *avail, int64_t ld_avail, float scale, const float *log_sum,
                       const float *entropy, const float *grad_logp, const float *grad_entropy, void *grad_logits,
                       int64_t ld_grad, void *hip_stream)
{
    const int rc = log_prob_check(dtype, R, V, logits, ld, avail, ld_avail, scale);
    if (rc) return rc;
    if (ld_grad < V) return MARL_ERR_BAD_DIM;
    if (grad_logits && grad_logits == logits && ld_grad != ld) return MARL_ERR_BAD_ARG;
    if (R == 0) return MARL_OK;
    if (!log_sum || !grad_logits || (grad_logp && !token) || (grad_entropy && !entropy)) return MARL_ERR_NULL;
    LogProbArgs p{};
    p.R = R; p.V = V;
    p.logits = logits; p.ld = ld; p.token = token; p.avail = avail; p.ld_avail = ld_avail; p.scale = scale; p.lowest = lowest_of(scale);
    p.in_log_sum = log_sum; p.in_entropy = entropy; p.grad_logp = grad_logp; p.grad_entropy = grad_entropy;
    p.grad_logits = grad_logits; p.ld_grad = ld_grad;
    return with_dtype(dtype, [&](auto e) { return run_backward<decltype(e)>(p, static_cast<hipStream_t>(hip_stream)); });
}

}  // extern "C"
