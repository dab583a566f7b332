// Rows of logits and their masks: how the operators on them read long rows and short ones, and how long rows are cut.
#pragma once
#include <algorithm>
#include <cmath>
#include <limits>

#include "device_math.h"
#include "operator_types.h"

namespace marl {

constexpr int kThreads = 256;
constexpr float kInf = __builtin_inff();

struct LogitRows {
    int R, V;
    const void *logits;
    int64_t ld;
    const uint8_t *avail;
    int64_t ld_avail;
    float scale;
    float lowest;                      // what is below it has a z of -infinity, and no probability
};

__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(kLog2e * v); }

__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// scale * logit, rounded on its own wherever it is used: the distance of the likeliest entry is exactly 0 (fused with the subtraction it
// would be what the maximum's rounding left out), so that a lone entry has log probability 0 and none comes out above it.
__device__ __forceinline__ float rounded(float scale, float logit)
{
#pragma clang fp contract(off)
    return scale * logit;
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

__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
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
    __device__ __forceinline__ Taken read(const LogitRows &p, int64_t first, int64_t row, bool there, int token, float (&held)[N])
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

// ---------------------------------------------------------------------------------- on the host
// Rows without a gap between them, and masks too.
inline bool rows_are_flat(const LogitRows &p) { return p.ld == p.V && (!p.avail || p.ld_avail == 0 || p.ld_avail == p.V); }

// The lowest finite logit whose product with the scale, rounded to fp32, is finite.
inline float lowest_of(float scale)
{
    const float least = std::numeric_limits<float>::lowest();
    if (scale <= 1.0f) return least;
    float v = least / scale;                                           // within a step of it
    while (!std::isfinite(scale * v)) v = std::nextafter(v, 0.0f);
    for (float w; std::isfinite(scale * (w = std::nextafter(v, least)));) v = w;
    return v;
}

inline int logit_rows_check(int dtype, int R, int V, const void *logits, int64_t ld, const uint8_t *avail, int64_t ld_avail, float scale)
{
    if (!known_dtype(dtype)) return MARL_ERR_BAD_DTYPE;
    if (R < 0 || V < 1 || V >= (1 << 30) || ld < V) return MARL_ERR_BAD_DIM;
    if (avail && ld_avail != 0 && ld_avail < V) return MARL_ERR_BAD_DIM;
    if (!std::isfinite(scale) || !(scale > 0.0f)) return MARL_ERR_BAD_ARG;
    return !logits && R > 0 ? MARL_ERR_NULL : MARL_OK;
}

// Parts of a long row: one per chunk if asked for, as with alternatives; otherwise as many as fill the chip (eight workgroups on each of
// 256 compute units), not less than a chunk each.
struct Cut { int parts, per; };
inline Cut cut_of(int R, int V, int chunk, bool one_each)
{
    const int chunks = (V + chunk - 1) / chunk;
    const int wanted = one_each ? chunks : (int)std::min<int64_t>(chunks, std::max<int64_t>(1, 2048 / std::max(R, 1)));
    const int per = (chunks + wanted - 1) / wanted;
    return {(chunks + per - 1) / per, per};
}

}  // namespace marl
