// Products of the Newton-Schulz iteration on the fp16 matrix pipe.
//
// Every matrix of the iteration is kept as two fp16 planes of its entries times 2^12: hi = fp16(v), lo = fp16(v - hi), whatever the type of
// the matrices.  The scale keeps lo above fp16's subnormals at the size that entries of large matrices have, and leaves room up
// to 16 (singular values end near 1.2).  D = A B^T with both operands adjacent along the summed index, so that both are read the
// same way; G and P are symmetric, and X is kept beside its transpose.
//
// A product is hi hi + hi lo + lo hi in fp32 accumulators; what is left out, lo lo, is 2^-22 of a term.  Planes alternate in blocks of 32
// of the summed index, [hi x 32][lo x 32].  (One plane is not enough for bf16 matrices either: it leaves 1.2e-3 to 2.8e-3 of the result, where
// its rounding to bf16 leaves 1.7e-3.)
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "operator_types.h"

namespace marl {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr float kPlaneScale = 4096.0f;

// D[m, n] = alpha sum_k A[m, k] B[n, k] + beta C[m, n], m < Mp, n < Np (multiples of 64: the matrices are padded with zeros).
// Strides and rows are in fp16 values; offset of (r, k) in planes: r ld + plane_at(k).
struct Product {
    const _Float16 *A, *B;
    int64_t a_batch, b_batch;
    int64_t lda, ldb;
    int Mp, Np, stages;               // stages of 64 fp16 values of a row: 32 of the summed index
    float alpha, beta;
    const _Float16 *C;                // [n][m], of scaled entries; used with beta != 0
    _Float16 *Dt;                     // [n][m]
    _Float16 *D;                      // [m][n] or NULL
    int64_t ldt, ldd, t_batch, d_batch;        // C lies as Dt
    int symmetric;                    // A is B: only tiles on and below the diagonal, D is the mirrored tile
    int tiles_m, tiles_n, tiles;      // tiles: of one batch member
    int splits;                       // parts of the sum, one workgroup each; > 1: accumulators go to `partial`
    float *partial;                   // [batch][tiles][splits][16 MT NT / 4][threads] x 4
    // The last product of an update writes the matrix itself, [rows][cols]: out = keep weights - rate D, or D without weights
    void *out;                        // NULL: planes
    const void *weights;
    int rows, cols, tall;             // tall: rows are m, otherwise rows are n
    float keep, rate;
};

__host__ __device__ __forceinline__ int plane_at(int k) { return (k >> 5) * 64 + (k & 31); }

// KW groups of WM x WN waves take the stages of the sum in turn and put their results together at the end: where there are fewer tiles
// than compute units, the time of a product is that of one workgroup's stages one after the other.
template <int WM_, int WN_, int MT_, int NT_, int BUFFERS_, int KW_ = 1>
struct TileShape {
    static constexpr int WM = WM_, WN = WN_, MT = MT_, NT = NT_, kBuffers = BUFFERS_, KW = KW_;
    static constexpr int kWaves = WM * WN, kTileThreads = kWaves * kWave, kThreads = KW * kTileThreads;
    static constexpr int TM = WM * MT * 32, TN = WN * NT * 32;
    static constexpr int kStage = (TM + TN) * 128;                     // bytes: 64 fp16 values of every row
    // staging of MB blocks below one another: fp32 values of a row of results, and bytes a wave for 32 columns of them
    static constexpr int pitch(int MB) { return 32 * MB + 4; }
    static constexpr int staging(int MB) { return 32 * pitch(MB) * 4; }
    static constexpr int kStaging = staging(MT);
    static constexpr int kQuads = 4 * MT * NT;                         // groups of four accumulators of a lane
    static constexpr int kJoining = (KW - 1) * kQuads * kTileThreads * 16;                 // bytes: what the groups behind the first hand over
    static constexpr int kMost = kWaves * kStaging > kJoining ? kWaves * kStaging : kJoining;
    static constexpr int kLds = kBuffers * KW * kStage > kMost ? kBuffers * KW * kStage : kMost;
};

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

// Tile (i, j) of a linear index.  Workgroups go round the eight dies in turn, so consecutive tiles are given to one die, and
// they walk down strips eight tiles wide, so that what a die works on at a time shares its operands.
__device__ __forceinline__ void tile_of(const Product &p, int id, int &i, int &j)
{
    if (p.symmetric) {
        i = (int)((sqrtf(8.0f * (float)id + 1.0f) - 1.0f) * 0.5f);
        while (i * (i + 1) / 2 > id) --i;
        while ((i + 1) * (i + 2) / 2 <= id) ++i;
        j = id - i * (i + 1) / 2;
        return;
    }
    const int strip = id / (8 * p.tiles_m), first = strip * 8, width = min(8, p.tiles_n - first);
    const int in = id - strip * 8 * p.tiles_m;
    i = in / width;
    j = first + in % width;
}

__device__ __forceinline__ int die_order(int id, int n)
{
    const int per = n / 8, rest = n % 8, die = id % 8;
    return die * per + min(die, rest) + id / 8;
}

__device__ __forceinline__ void wave_meets()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Eight results along a row as planes.
__device__ __forceinline__ void put_planes(_Float16 *to, const float (&v)[8])
{
    half8 h, l;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        h[e] = (_Float16)v[e];
        l[e] = (_Float16)(v[e] - (float)h[e]);
    }
    *reinterpret_cast<half8 *>(to) = h;
    *reinterpret_cast<half8 *>(to + 32) = l;
}

// Eight results along row r, from column c, of the matrix itself.
template <typename E>
__device__ __forceinline__ void put_out(const Product &p, int64_t batch, int r, int c, const float (&v)[8])
{
    if (r >= p.rows) return;
    const int64_t at = (batch * p.rows + r) * p.cols + c;
    const E *w = static_cast<const E *>(p.weights);
    E *out = static_cast<E *>(p.out);
    const float rate = p.rate * (1.0f / kPlaneScale);
    auto one = [&](float x, float was) { return w ? p.keep * was - rate * x : x * (1.0f / kPlaneScale); };
    typedef E Eight __attribute__((ext_vector_type(8), aligned(sizeof(E))));
    if (c + 8 <= p.cols) {
        Eight o, was;
        if (w) was = *reinterpret_cast<const Eight *>(w + at);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = from_f32<E>(one(v[e], w ? to_f32((E)was[e]) : 0.0f));
        *reinterpret_cast<Eight *>(out + at) = o;
    } else {
        for (int e = 0; e < 8; ++e)
            if (c + e < p.cols) out[at + e] = from_f32<E>(one(v[e], w ? to_f32(w[at + e]) : 0.0f));
    }
}

// What becomes of a tile's accumulators.  Through shared memory, 32 columns at a time and each wave for itself, so that memory is
// read and written along rows: once in the order [n][m], where C is added, and once in the order [m][n].  MB x NB of
// the wave's MT x NT blocks of 32 x 32, from (mb0, nb0) on.
template <class S, typename E, int MB, int NB>
__device__ __forceinline__ void put_tile(const Product &p, int64_t batch, int m0, int n0, int mb0, int nb0, bool diagonal, floatx16 (&acc)[MB][NB], char *lds)
{
    constexpr int kPitch = S::pitch(MB), kAlong = MB * 4;               // kAlong: eights of a row of m
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int wm = m0 + (wave / S::WN) * S::MT * 32 + mb0 * 32, wn = n0 + (wave % S::WN) * S::NT * 32 + nb0 * 32;
    float *stage = reinterpret_cast<float *>(lds + wave * S::staging(MB));
    const _Float16 *C = p.C + batch * p.t_batch;
    const bool transposed = p.out ? p.tall != 0 : p.D && !diagonal;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        wave_meets();
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<floatx4 *>(stage + (lane & 31) * kPitch + mb * 32 + 8 * q + 4 * (lane >> 5)) =
                    floatx4{acc[mb][nb][4 * q], acc[mb][nb][4 * q + 1], acc[mb][nb][4 * q + 2], acc[mb][nb][4 * q + 3]};
        wave_meets();
#pragma unroll 4
        for (int k = lane; k < 32 * kAlong; k += kWave) {
            const int col = k / kAlong, along = k % kAlong * 8, n = wn + nb * 32 + col, m = wm + along;
            if (n >= p.Np || m >= p.Mp) continue;
            float *at = stage + col * kPitch + along, v[8];
            const int64_t lies = n * p.ldt + plane_at(m);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = p.alpha * at[e];
            if (p.beta != 0.0f) {
                const half8 h = *reinterpret_cast<const half8 *>(C + lies), l = *reinterpret_cast<const half8 *>(C + lies + 32);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = fmaf(p.beta, (float)h[e] + (float)l[e], v[e]);
            }
            if (transposed) {
#pragma unroll
                for (int e = 0; e < 8; ++e) at[e] = v[e];
            }
            if (p.out) {
                if (!p.tall) put_out<E>(p, batch, n, m, v);
            } else {
                put_planes(p.Dt + batch * p.t_batch + lies, v);
            }
        }
        if (!transposed) continue;
        wave_meets();
#pragma unroll 2
        for (int k = lane; k < 32 * MB * 4; k += kWave) {              // row k / 4, eight columns
            const int row = k / 4, col = k % 4 * 8, m = wm + row, n = wn + nb * 32 + col;
            if (n >= p.Np || m >= p.Mp) continue;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = stage[(col + e) * kPitch + row];
            if (p.out) {
                put_out<E>(p, batch, m, n, v);
            } else {
                const int64_t lies = m * p.ldd + plane_at(n);
                put_planes(p.D + batch * p.d_batch + lies, v);
            }
        }
    }
}

template <class S, typename E>
__global__ __launch_bounds__(S::kThreads) void product_kernel(Product p)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int MT = S::MT, NT = S::NT, TM = S::TM, TN = S::TN;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave % S::kWaves;
    const int group = S::KW == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / S::kTileThreads);
    const int units = p.tiles * p.splits;
    const int unit = die_order(blockIdx.x, units), tile = unit % p.tiles, split = unit / p.tiles;
    const int64_t batch = blockIdx.y;
    int ti, tj;
    tile_of(p, tile, ti, tj);
    const int m0 = ti * TM, n0 = tj * TN;
    const int k_begin = (int)((int64_t)split * p.stages / p.splits), k_end = (int)((int64_t)(split + 1) * p.stages / p.splits);

    // A wave's load brings eight rows of 128 bytes; chunk c of row r goes to place c ^ (r / 2 & 7), so that sixteen lanes reading the
    // same chunk of neighbouring rows meet all 64 banks (with c ^ (r & 7) half of the cycles were conflicts).  The place in shared memory
    // is fixed by the lane, so the lane asks for the chunk that belongs there.
    constexpr int kLoadsA = TM / 8 / S::kWaves, kLoadsB = TN / 8 / S::kWaves;
    static_assert(kLoadsA * 8 * S::kWaves == TM && kLoadsB * 8 * S::kWaves == TN && S::kWaves % 2 == 0, "");
    const int sub = lane >> 3, chunk = (lane & 7) ^ ((wave & 1) * 4 + sub / 2);
    const _Float16 *from_a[kLoadsA], *from_b[kLoadsB];
#pragma unroll
    for (int q = 0; q < kLoadsA; ++q)
        from_a[q] = p.A + batch * p.a_batch + (int64_t)min(m0 + (q * S::kWaves + wave) * 8 + sub, p.Mp - 1) * p.lda + chunk * 8;
#pragma unroll
    for (int q = 0; q < kLoadsB; ++q)
        from_b[q] = p.B + batch * p.b_batch + (int64_t)min(n0 + (q * S::kWaves + wave) * 8 + sub, p.Np - 1) * p.ldb + chunk * 8;
    const int turns = (k_end - k_begin + S::KW - 1) / S::KW;           // stages of a group; the last may be one behind the end
    auto load = [&](int turn, int buffer) {
        char *to = lds + (buffer * S::KW + group) * S::kStage;
        const int k = min(k_begin + min(turn, turns - 1) * S::KW + group, k_end - 1);
#pragma unroll
        for (int q = 0; q < kLoadsA; ++q)
            __builtin_amdgcn_global_load_lds((global_void *)(from_a[q] + (int64_t)k * 64), (lds_void *)(to + (q * S::kWaves + wave) * 1024), 16, 0, 0);
#pragma unroll
        for (int q = 0; q < kLoadsB; ++q)
            __builtin_amdgcn_global_load_lds((global_void *)(from_b[q] + (int64_t)k * 64), (lds_void *)(to + TM * 128 + (q * S::kWaves + wave) * 1024), 16, 0, 0);
    };
    floatx16 acc[MT][NT];
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[a][b][e] = 0.0f;

    // A matrix instruction cuts its products off where the sum so far ends, so a long sum of squares, the diagonal of G, loses a part that grows
    // with its length.  Where there are registers for it, 256 terms are summed by themselves and added to the rest in fp32 (20 x 4000 fp32:
    // relative error 2.9e-6 in one sum, 1.4e-6 so; 1000 x 1000 1.7e-6 and 0.9e-6; fp32 products of an elementary form leave
    // 1.15e-6 and 2.5e-6.  Three of 1000 x 333 take 4 % longer for it).
    constexpr bool kBySpans = MT * NT <= 4;
    constexpr int kSpan = 8 / S::KW;                                   // stages
    floatx16 total[kBySpans ? MT : 1][kBySpans ? NT : 1];
    auto add_span = [&](bool first) {
        if constexpr (kBySpans) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int u = 0; u < NT; ++u)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        total[t][u][e] = first ? 0.0f : total[t][u][e] + acc[t][u][e];
                        acc[t][u][e] = 0.0f;
                    }
        }
    };
    add_span(true);
    const int row = lane & 31, high = lane >> 5;
    const char *read_a = lds + group * S::kStage + ((wave / S::WN) * MT * 32 + row) * 128, *read_b = lds + group * S::kStage + TM * 128 + ((wave % S::WN) * NT * 32 + row) * 128;
    auto frag = [&](const char *base, int block, int c) {
        return *reinterpret_cast<const half8 *>(base + block * 32 * 128 + ((c ^ (row / 2 & 7)) << 4));
    };
    // Fragments are read one step (16 of the summed index) ahead of the products that take them, so that shared memory and the matrix
    // pipe work at the same time; the first step of the next stage is read behind the barrier that stands before the last
    // step's products.  By then the stage in hand has been read to its end, so its buffer takes the stage after the next.
    constexpr int kInStage = 2;
    half8 a[2][2][MT], b[2][2][NT];
    auto read = [&](int set, int buffer, int j) {
        const char *ra = read_a + buffer * (S::KW * S::kStage), *rb = read_b + buffer * (S::KW * S::kStage);
#pragma unroll
        for (int pl = 0; pl < 2; ++pl) {
#pragma unroll
            for (int t = 0; t < MT; ++t) a[set][pl][t] = frag(ra, t, 4 * pl + 2 * j + high);
#pragma unroll
            for (int t = 0; t < NT; ++t) b[set][pl][t] = frag(rb, t, 4 * pl + 2 * j + high);
        }
    };
    // The oldest stage on its way has arrived: this wave's part of it, then everybody's.  A wave's loads return in order, kLoads
    // a stage; the later stages stay on their way.
    constexpr int kLoads = kLoadsA + kLoadsB;
    auto arrive = [&] { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((S::kBuffers - 2) * kLoads) : "memory"); };
    constexpr int kReads = 2 * (MT + NT), kProducts = 3 * MT * NT;
    auto products = [&](int set) {
#pragma unroll
        for (int part = 0; part < 3; ++part)           // hi hi, hi lo, lo hi
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int u = 0; u < NT; ++u)
                    acc[t][u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[set][part == 2][t], b[set][part == 1][u], acc[t][u], 0, 0, 0);
    };
    // Products, then one read, in turn: reads in a row would hold up the products behind them until shared memory took them.  The
    // loads of a stage come first (they write shared memory, so no read passes them), a product between them.
    auto in_turn = [&](auto loads) {
        constexpr int kFirst = decltype(loads)::value ? kLoads : 0, kEach = (kProducts - kFirst) / kReads > 0 ? (kProducts - kFirst) / kReads : 1;
#pragma unroll
        for (int q = 0; q < kFirst; ++q) {
            __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
#pragma unroll
        for (int q = 0; q < kReads; ++q) {
            __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, kProducts, 0);
    };
#pragma unroll
    for (int q = 0; q < S::kBuffers - 1; ++q) load(q, q);              // (every part has a stage at least)
    arrive();
    load(S::kBuffers - 1, S::kBuffers - 1);
    read(0, 0, 0);
    int buffer = 0;
    for (int turn = 0; turn + 1 < turns; ++turn) {
        const int next = buffer + 1 == S::kBuffers ? 0 : buffer + 1;
#pragma unroll
        for (int j = 0; j < kInStage; ++j) {
            if (j + 1 < kInStage) {
                read((j + 1) & 1, buffer, j + 1);
            } else {
                arrive();
                load(turn + S::kBuffers, buffer);                      // (behind the last stage: once more, and not read)
                read((j + 1) & 1, next, 0);
            }
            products(j & 1);
            if (j + 1 < kInStage) in_turn(std::false_type{});
            else in_turn(std::true_type{});
        }
        buffer = next;
        if constexpr (kBySpans)
            if (turn % kSpan == kSpan - 1) add_span(false);
    }
    if (S::KW == 1 || k_begin + (turns - 1) * S::KW + group < k_end) {
#pragma unroll
        for (int j = 0; j < kInStage; ++j) {
            if (j + 1 < kInStage) read((j + 1) & 1, buffer, j + 1);
            products(j & 1);
        }
    }
    if constexpr (kBySpans) {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[t][u][e] += total[t][u][e];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                   // nothing may still be on its way into the buffers
    if constexpr (S::KW > 1) {                                         // the groups' sums, in order
        __syncthreads();
        floatx4 *to = reinterpret_cast<floatx4 *>(lds) + threadIdx.x % S::kTileThreads;
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int b = 0; b < NT; ++b)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int quad = (a * NT + b) * 4 + q;
                    if (group > 0)
                        to[((group - 1) * S::kQuads + quad) * S::kTileThreads] = floatx4{acc[a][b][4 * q], acc[a][b][4 * q + 1], acc[a][b][4 * q + 2], acc[a][b][4 * q + 3]};
                }
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int a = 0; a < MT; ++a)
#pragma unroll
                for (int b = 0; b < NT; ++b)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int g = 0; g < S::KW - 1; ++g) {
                            const floatx4 more = to[(g * S::kQuads + (a * NT + b) * 4 + q) * S::kTileThreads];
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[a][b][4 * q + e] += more[e];
                        }
        }
    }
    __syncthreads();                                                   // the buffers become staging room
    if (group > 0) return;
    if (p.splits > 1) {
        floatx4 *to = reinterpret_cast<floatx4 *>(p.partial) + ((batch * p.tiles + tile) * p.splits + split) * (S::kQuads * S::kTileThreads) + threadIdx.x;
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int b = 0; b < NT; ++b)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    to[((a * NT + b) * 4 + q) * S::kTileThreads] = floatx4{acc[a][b][4 * q], acc[a][b][4 * q + 1], acc[a][b][4 * q + 2], acc[a][b][4 * q + 3]};
        return;
    }
    put_tile<S, E, MT, NT>(p, batch, m0, n0, 0, 0, p.symmetric && ti == tj, acc, lds);
}

// Sums the parts of a tile, in order, and finishes it.  A workgroup takes two of each wave's blocks, so that there are several for a tile:
// the parts of a split product are few tiles, and one workgroup each left half of the chip and most of its memory idle.
template <class S> constexpr int kJoinBlocks = S::MT < 2 ? S::MT : 2;
template <class S, typename E>
__global__ __launch_bounds__(S::kTileThreads) void join_kernel(Product p)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int MT = kJoinBlocks<S>;
    const int64_t batch = blockIdx.y;
    const int tile = blockIdx.x, nb = blockIdx.z % S::NT, mb = blockIdx.z / S::NT * MT;
    int ti, tj;
    tile_of(p, tile, ti, tj);
    const floatx4 *from = reinterpret_cast<const floatx4 *>(p.partial) + (batch * p.tiles + tile) * p.splits * (S::kQuads * S::kTileThreads) + threadIdx.x;
    floatx4 sum[MT][4];
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int q = 0; q < 4; ++q) sum[a][q] = floatx4{0, 0, 0, 0};
    for (int s = 0; s < p.splits; ++s)
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int q = 0; q < 4; ++q) sum[a][q] += from[(s * S::kQuads + ((mb + a) * S::NT + nb) * 4 + q) * S::kTileThreads];
    floatx16 acc[MT][1];
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[a][0][4 * q + e] = sum[a][q][e];
    put_tile<S, E, MT, 1>(p, batch, ti * S::TM, tj * S::TN, mb, nb, p.symmetric && ti == tj, acc, lds);
}

}  // namespace marl
