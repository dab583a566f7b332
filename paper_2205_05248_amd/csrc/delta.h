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
#include <type_traits>

#include "operator_types.h"

namespace marl {

constexpr int kSteps = 64;                             // of a chunk
constexpr int kDeltaThreads = 256;                     // four waves; wave w has rows 16 w on of a chunk

typedef float Acc __attribute__((ext_vector_type(4)));

// Products run on the bf16 matrix pipe on sums of bf16 planes: a plane holds what the planes before it left, rounded to 8 bits, so that
// three hold 24 of a value's bits.  bf16 elements are one plane, fp16 two, fp32 three, all exactly.  States, matrices and steps are
// three whatever the elements' type: a 16-bit result too can be what large numbers leave of each other.  Of the products of
// planes those are formed that are not below the smallest kept: six of three by three.  The fp32
// matrix instructions would be 16 times slower, and fp16 planes, of which two would do, need every column scaled to their range.
typedef __bf16 Frag __attribute__((ext_vector_type(8)));
typedef __bf16 Four __attribute__((ext_vector_type(4)));
template <typename E> constexpr int kExact = sizeof(E) == 4 ? 3 : std::is_same<E, _Float16>::value ? 2 : 1;

struct ChunkGates {
    double G[kSteps];
    float f[kSteps], t[kSteps], beta[kSteps];          // t: -1 in padding
    float whole;                                       // f of the last step
    int bad;                                           // the rows of K or Q, N or P hold an infinity or NaN
    unsigned long long starts, live;                   // bit i: step i starts a sequence; is none of the padding
    int pad[26];
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
    // workspace.  Matrices in the order in which the matrix instructions take them: tiles of 16 rows by 32 columns, plane by plane, a lane's
    // eight entries (row l % 16, columns l / 16 * 8 on) adjacent, so that a wave reads and writes 1 KB at a time.
    Frag *K, *Q, *KT, *QT;                             // per (b, key head, chunk): rows, and transposed; QT null without keep
    Frag *N, *P, *NT, *PT;                             // per (b, value head, chunk); NT and PT null without keep
    ChunkGates *gates;                                 // per (b, value head, chunk), as all that follow
    // with keys and values padded, so that nothing asks where a row ends; null without keep
    float *S, *M;                                      // [DK,DV] before the chunk, [64,DV]
    float *D, *Y;                                      // [DK,DV] adjoint behind the chunk, [64,DV]
};
constexpr int padded_keys(int Dk) { return Dk <= 32 ? 32 : Dk <= 64 ? 64 : 128; }
__host__ __device__ constexpr int padded_values(int Dv) { return (Dv + 31) / 32 * 32; }

// Fragments of one matrix: of the keys of a chunk (padded to DK), and of N and its kind.
constexpr int key_frags(int DK, int planes) { return kSteps / 16 * (DK / 32) * planes * kWave; }
constexpr int square_frags(int planes) { return kSteps / 16 * 2 * planes * kWave; }
// The lane's fragment of tile (16 rows), step (32 columns) and plane.
__device__ __forceinline__ int frag_at(int tile, int step, int plane, int steps, int planes)
{
    return ((tile * steps + step) * planes + plane) * kWave + (int)threadIdx.x % kWave;
}

__device__ __forceinline__ float max_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }      // NaN stays
__device__ __forceinline__ float decay_of(double d) { return max_of(expf((float)d), 1.17549435e-38f); }

// Sequences of a chunk that have started up to and with step i.
__device__ __forceinline__ int part_of(unsigned long long starts, int i) { return __popcll(starts << (63 - i)); }
__device__ __forceinline__ bool bit_of(unsigned long long bits, int i) { return bits >> i & 1; }
// Whether step j hands anything to step i >= j.
__device__ __forceinline__ bool joined(unsigned long long starts, int i, int j) { return part_of(starts, i) == part_of(starts, j); }
// Steps of i's sequence up to and with i; from i on.
__device__ __forceinline__ unsigned long long upto(unsigned long long starts, int i)
{
    const unsigned long long low = ~0ull >> (63 - i), before = starts & low;
    return before ? low & ~0ull << (63 - __clzll((long long)before)) : low;
}
__device__ __forceinline__ unsigned long long from(unsigned long long starts, int i)
{
    const unsigned long long high = ~0ull << i, behind = starts & high & ~(1ull << i);
    return behind ? high & (behind & -behind) - 1 : high;
}

// Planes of four values.  (Pairs: one instruction converts two.)
template <int N>
__device__ __forceinline__ void split(Acc v, Four (&out)[N])
{
    typedef __bf16 Two __attribute__((ext_vector_type(2)));
    typedef float Pair __attribute__((ext_vector_type(2)));
    Pair x{v[0], v[1]}, y{v[2], v[3]};
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const Two low = __builtin_convertvector(x, Two), high = __builtin_convertvector(y, Two);
        out[n] = __builtin_shufflevector(low, high, 0, 1, 2, 3);
        if (n + 1 < N) {
            x -= __builtin_convertvector(low, Pair);
            y -= __builtin_convertvector(high, Pair);
        }
    }
}
template <int N>
__device__ __forceinline__ void split(const float *v, Frag (&out)[N])
{
    Four low[N], high[N];
    split(Acc{v[0], v[1], v[2], v[3]}, low);
    split(Acc{v[4], v[5], v[6], v[7]}, high);
#pragma unroll
    for (int n = 0; n < N; ++n) out[n] = __builtin_shufflevector(low[n], high[n], 0, 1, 2, 3, 4, 5, 6, 7);
}

// c + a b on a 16 x 32 by 32 x 16 tile, the smallest products first; ORDER: the largest sum of plane numbers that counts.  Lane l holds rows
// l / 16 * 4 .. + 4 of column l % 16 of the result.
template <int PA, int PB, int ORDER = (PA > PB ? PA : PB) - 1>
__device__ __forceinline__ Acc multiply(const Frag (&a)[PA], const Frag (&b)[PB], Acc c)
{
#pragma unroll
    for (int s = ORDER; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (s - i >= 0 && s - i < PB) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[s - i], c, 0, 0, 0);
    return c;
}

// The same with a sum of its own for the products of every size: none waits for another's, and small ones are not rounded to the size of large ones.
template <int ORDER> struct Sums { Acc c[ORDER + 1] = {}; };
template <int PA, int PB, int ORDER>
__device__ __forceinline__ void multiply_into(Sums<ORDER> &sums, const Frag (&a)[PA], const Frag (&b)[PB])
{
#pragma unroll
    for (int s = ORDER; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (s - i >= 0 && s - i < PB) sums.c[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[s - i], sums.c[s], 0, 0, 0);
}
template <int ORDER>
__device__ __forceinline__ Acc total(const Sums<ORDER> &sums)
{
    Acc v = sums.c[ORDER];
#pragma unroll
    for (int s = ORDER - 1; s >= 0; --s) v += sums.c[s];
    return v;
}

// The same over 64 columns k without the matrix pipe, for chunks that hold an infinity or NaN: only the k in pass[r] take part in the lane's
// r-th row.  a: the matrix's fragments; b: the lane's column, planes `plane` apart.
template <int PA, int PB>
__device__ __forceinline__ Acc careful_multiply(Acc c, const Frag *a, int tile, const __bf16 *b, int plane, const unsigned long long (&pass)[4])
{
    const int group = threadIdx.x % kWave / 16;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        float v = c[r];
#pragma unroll 1
        for (int k = 0; k < kSteps; ++k) {
            if (!bit_of(pass[r], k)) continue;
            float x = 0.0f, y = 0.0f;
            for (int n = PA - 1; n >= 0; --n)
                x += (float)reinterpret_cast<const __bf16 *>(a)[(((tile * 2 + k / 32) * PA + n) * kWave + group * 4 + r + k % 32 / 8 * 16) * 8 + k % 8];
            for (int n = PB - 1; n >= 0; --n) y += (float)b[n * plane + k];
            v = fmaf(x, y, v);
        }
        c[r] = v;
    }
    return c;
}
// What planes can hold: the first one of a value beyond 3.39e38 is rounded to infinity.  A NaN does not fit either.
__device__ __forceinline__ bool fits_planes(float size) { return size < 3.36e38f; }
__device__ __forceinline__ bool all_finite(Acc a)      // (and fit planes)
{
    const Acc z = a * 1.0126f * 0.0f;
    return (z[0] + z[1]) + (z[2] + z[3]) == 0.0f;
}

// c + a b on 16 x 16 tiles in fp32: a(row, k), b(k, col) give one entry each.  All entries are asked for before the first is used.
template <class FA, class FB>
__device__ __forceinline__ Acc product(Acc c, FA &&a, FB &&b)
{
    const int lane = threadIdx.x % kWave, at = lane % 16, group = lane / 16;
    float x[4], y[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) x[s] = a(at, s * 4 + group), y[s] = b(s * 4 + group, at);
#pragma unroll
    for (int s = 0; s < 4; ++s) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[s], y[s], c, 0, 0, 0);
    return c;
}

// Row of the elements of step t of sequence b and head h.
template <typename E>
__device__ __forceinline__ const E *row_at(const void *base, int64_t ld, int64_t b, int T, int t, int h, int D)
{
    return static_cast<const E *>(base) + (b * T + t) * ld + (int64_t)h * D;
}

// NT adjacent columns of a row, 0 behind the last; and back.  16-byte alignment is not needed, nor any above the element's.
template <typename E, int NT>
__device__ __forceinline__ void read_columns(const E *row, int col, int D, float (&to)[NT])
{
    typedef E Vec __attribute__((ext_vector_type(NT)));
    typedef Vec Loose __attribute__((aligned(sizeof(E))));
    if (col + NT <= D) {
        const Vec v = *reinterpret_cast<const Loose *>(row + col);
#pragma unroll
        for (int n = 0; n < NT; ++n) to[n] = to_f32(v[n]);
    } else {
#pragma unroll
        for (int n = 0; n < NT; ++n) to[n] = col + n < D ? to_f32(row[col + n]) : 0.0f;
    }
}
template <typename E, int NT>
__device__ __forceinline__ void write_columns(E *row, int col, int D, const float (&from)[NT])
{
    typedef E Vec __attribute__((ext_vector_type(NT)));
    typedef Vec Loose __attribute__((aligned(sizeof(E))));
    if (col + NT <= D) {
        Vec v;
#pragma unroll
        for (int n = 0; n < NT; ++n) v[n] = from_f32<E>(from[n]);
        *reinterpret_cast<Loose *>(row + col) = v;
    } else {
#pragma unroll
        for (int n = 0; n < NT; ++n)
            if (col + n < D) row[col + n] = from_f32<E>(from[n]);
    }
}

// A 0 that the compiler does not know.  Added to an address that is the same for all lanes it keeps the load off the scalar unit, where a load
// still under way delays every access to shared memory.
__device__ __forceinline__ int hidden_zero()
{
    int zero;
    asm volatile("v_mov_b32 %0, 0" : "=v"(zero));
    return zero;
}

__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); }

// Reads of a record at an offset in bytes that fits 32 bits: uniform base, one register a lane.
template <typename V>
__device__ __forceinline__ V read_at(const void *base, unsigned offset) { return *reinterpret_cast<const V *>(static_cast<const char *>(base) + offset); }

// The fragments of a matrix: the number of one is the same for all lanes of a wave and goes through a scalar register.
struct FragReader {
    __amdgpu_buffer_rsrc_t buffer;
    __device__ __forceinline__ FragReader(const Frag *record) : buffer(__builtin_amdgcn_make_buffer_rsrc(const_cast<Frag *>(record), 0, -1, 0x00020000)) {}
    __device__ __forceinline__ Frag at(int tile, int step, int plane, int steps, int planes) const
    {
        const int number = (tile * steps + step) * planes + plane;
        return __builtin_bit_cast(Frag, __builtin_amdgcn_raw_buffer_load_b128(buffer, (int)threadIdx.x % kWave * 16, number * 1024, 0));
    }
};

// NT adjacent columns of a row as they lie in memory: loaded at once, whatever the row's end, and looked at later, so that the load can be on its way
// meanwhile.  (With a conversion or a branch behind the load every row of the next chunk was waited for where it was asked for.)
template <typename E, int NT>
struct Columns {
    typedef E Vec __attribute__((ext_vector_type(NT)));
    typedef Vec Loose __attribute__((aligned(sizeof(E))));
    Vec raw;
    // offset: of the row's column min(col, D - NT), in bytes from `base`.  D >= NT: two tiles are taken of more than 16 columns only
    __device__ __forceinline__ void load(const E *base, unsigned offset) { raw = read_at<Loose>(base, offset); }
    __device__ __forceinline__ float at(int n, int col, int D) const
    {
        const float own = to_f32(raw[n]), last = to_f32(raw[NT - 1]);
        return col + NT <= D ? own : col + n == D - 1 ? last : 0.0f;
    }
};

// Rows of a chunk's results, written without a branch: what lies behind the last step or column goes to an offset that the descriptor does not
// cover.  (Behind a branch the compiler cannot count the stores under way, and waits for them with the next chunk's loads.)  Row distances are
// below 2^24, so that 64 rows are covered by 32 bits.
constexpr int kRawBuffer = 0x00020000;
template <typename E, int NT>
struct RowsOut {
    __amdgpu_buffer_rsrc_t buffer;
    unsigned ld;
    int rows, Dv;
    bool pairs;
    __device__ __forceinline__ RowsOut(const DeltaArgs &p, void *base, int64_t ld_, int64_t b, int chunk, int h)
        : ld((unsigned)ld_), rows(min(kSteps, p.T - chunk * kSteps)), Dv(p.Dv)
    {
        E *first = const_cast<E *>(row_at<E>(base, ld_, b, p.T, chunk * kSteps, h, Dv));
        buffer = __builtin_amdgcn_make_buffer_rsrc(first, 0, (int)((ld * (unsigned)(rows - 1) + (unsigned)Dv) * (unsigned)sizeof(E)), kRawBuffer);
        pairs = sizeof(E) == 4 ? Dv % 2 == 0 : Dv % 2 == 0 && ld % 2 == 0 && (reinterpret_cast<uintptr_t>(base) & 3) == 0;
    }
    __device__ __forceinline__ void put(int row, int col, const float (&v)[NT]) const
    {
        typedef unsigned U2 __attribute__((ext_vector_type(2)));
        typedef E Vec __attribute__((ext_vector_type(NT)));
        const unsigned at = (ld * (unsigned)row + (unsigned)col) * (unsigned)sizeof(E), none = 0xfffffff0u;
        Vec w;
#pragma unroll
        for (int n = 0; n < NT; ++n) w[n] = from_f32<E>(v[n]);
        if constexpr (NT == 2) {
            if (pairs) {
                const unsigned to = row < rows && col < Dv ? at : none;
                if constexpr (sizeof(E) == 4) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(U2, w), buffer, to, 0, 0);
                else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, w), buffer, to, 0, 0);
                return;
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const unsigned to = row < rows && col + n < Dv ? at + n * (unsigned)sizeof(E) : none;
            if constexpr (sizeof(E) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, (float)w[n]), buffer, to, 0, 0);
            else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, (E)w[n]), buffer, to, 0, 0);
        }
    }
};

// The head and the first column of a workgroup on its way through the chunks.  Workgroups go to the eight dies in turn: those of a head, which
// read the same fragments, are given to one die.  head = -1: nothing to do.
struct Place { int64_t head; int first; };
__device__ __forceinline__ Place place_of(int64_t heads, int Dv, int columns)
{
    const int blocks = padded_values(Dv) / columns;
    const int64_t all = heads * blocks, each = (all + 7) / 8, at = (int64_t)(blockIdx.x % 8) * each + blockIdx.x / 8;
    return at < all && blockIdx.x / 8 < each ? Place{at / blocks, (int)(at % blocks) * columns} : Place{-1, 0};
}
inline unsigned places(int64_t heads, int Dv, int columns) { return (unsigned)((heads * (padded_values(Dv) / columns) + 7) / 8 * 8); }

// Whether a workgroup takes two tiles of columns: every fragment is read once for both, for half as many waves on a compute unit.  It needs more than
// two columns a lane can hold, and workgroups for the whole chip: one a compute unit where the keys' planes fill a wave's registers anyway, else two; where
// one tile alone leaves no room for a second workgroup, half of them, for as soon as there are more tiles than compute units some have two in turn.
// 8 | 32 sequences of 512 steps, 16 heads, 64 columns (256 | 1024 workgroups of two tiles), us with one and two, forward with keep and backward:
//   128 keys, bf16  60, 53 | 221, 206   70, 55 | 252, 204       64 keys, bf16  43, 38 | 169, 150   43, 42 | 161, 155
//   128 keys, fp32 108, 79 | 387, 305  103, 82 | 390, 303       64 keys, fp32  63, 50 | 231, 202   74, 52 | 276, 200
//    32 keys, bf16  38, 34 | 158, 123   34, 49 | 153, 137       32 keys, fp32  49, 59 | 191, 176   50, 102 | 191, 404
// 3 sequences, 11 heads, 128 columns (132 workgroups of two tiles), 128 keys: bf16 35, 43 and 44, 45; fp16 61, 48 and 70, 53; fp32 73, 59 and 78, 64.
// (backward with 32 keys two tiles spill, and are not taken.)
template <typename E, int DK>
inline bool wide_columns(const DeltaArgs &p)
{
    return p.Dv > 16 && (int64_t)p.B * p.Hv * (padded_values(p.Dv) / 32) >= (kExact<E> * DK >= 256 ? 129 : kExact<E> * DK >= 128 ? 256 : 512);
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
