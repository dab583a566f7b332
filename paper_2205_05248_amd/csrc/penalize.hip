// Penalties for repeated tokens, biases and a grammar's mask on rows of logits.  A workgroup takes a piece of a row: it counts the
// row's history in shared memory for the places of its piece and then passes the piece through once.  Bound by the bytes of the logits, read
// and written; every piece reads the history again, from the second-level cache.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "logit_rows.h"

namespace marl {
namespace {

constexpr int kMostBiases = 1024;

struct PenalizeArgs {
    int R, V, L, M, pieces;
    const void *logits;
    int64_t ld;
    const int32_t *history;
    int64_t ld_history;
    const int32_t *length, *prompt;
    const float *repetition, *presence, *frequency;
    const int32_t *bias_id;
    const float *bias_value;
    const uint32_t *allowed;
    int64_t ld_allowed;
    void *out;
    int64_t ld_out;
};

constexpr unsigned kSeen = 0x80000000u, kBiased = 0x40000000u, kCount = 0x3fffffffu;

// A place's word: whether it was seen, whether it has a bias, and how often it was generated (L < 2^24).
template <typename E, int THREADS, int PIECE>
__global__ __launch_bounds__(THREADS) void penalize_kernel(PenalizeArgs p)
{
    typedef Piece<E> P;
    constexpr int V = P::V;
    __shared__ __attribute__((aligned(16))) unsigned words[PIECE];
    const int64_t row = blockIdx.x / p.pieces;
    const int piece = blockIdx.x % p.pieces;
    const E *l = static_cast<const E *>(p.logits) + row * p.ld;
    E *out = static_cast<E *>(p.out) + row * p.ld_out;
    const int skew = skew_of(out);                                     // entry j of the row is skew + j
    const int n = p.V + skew, begin = piece * PIECE, end = min(begin + PIECE, n);
    const int length = p.length ? min(max(p.length[row], 0), p.L) : p.L;
    const int prompt = p.prompt ? min(max(p.prompt[row], 0), length) : 0;
    const bool counts = length > 0 || p.M > 0;
    if (counts) {
        for (int w = threadIdx.x * 4; w < end - begin; w += THREADS * 4) *reinterpret_cast<uint4 *>(words + w) = make_uint4(0, 0, 0, 0);
        __syncthreads();
        const int32_t *history = p.history + row * p.ld_history;
        for (int t = threadIdx.x; t < length; t += THREADS) {
            const int id = history[t];
            const int at = id + skew - begin;                          // no place of the piece if the id is none of the row
            if (id >= 0 && id < p.V && at >= 0 && at < end - begin) {
                atomicOr(&words[at], kSeen);
                if (t >= prompt) atomicAdd(&words[at], 1u);
            }
        }
        for (int m = threadIdx.x; m < p.M; m += THREADS) {
            const int id = p.bias_id[row * p.M + m];
            const int at = id + skew - begin;
            if (id >= 0 && id < p.V && at >= 0 && at < end - begin) atomicOr(&words[at], kBiased);
        }
        __syncthreads();
    }
    const float rho = p.repetition ? p.repetition[row] : 1.0f, presence = p.presence ? p.presence[row] : 0.0f;
    const float frequency = p.frequency ? p.frequency[row] : 0.0f;
    const uint32_t *allowed = p.allowed ? p.allowed + row * p.ld_allowed : nullptr;
    l -= skew;
    out -= skew;
    auto edit = [&](float z, unsigned word, int j) {
        if (word & kSeen) z = z > 0.0f ? z / rho : z * rho;
        const unsigned c = word & kCount;
        if (c) z = (z - presence) - frequency * (float)c;
        if (word & kBiased)
            for (int m = 0; m < p.M; ++m)                              // in their order, whichever thread set the bit
                if (p.bias_id[row * p.M + m] == j - skew) z += p.bias_value[row * p.M + m];
        return z;
    };
    // bits of the V places from entry j - skew of the row on
    auto bits_of = [&](int j) {
        const int e = j - skew, last = (p.V - 1) / 32;
        const int low = max(e, 0);
        const uint64_t pair = (uint64_t)allowed[min(low / 32 + 1, last)] << 32 | allowed[min(low / 32, last)];
        const unsigned bits = (unsigned)(pair >> (low % 32));
        return e < 0 ? bits << min(-e, 31) : bits;                     // (before the row nothing is written)
    };
    for (int j = begin + (int)threadIdx.x * V; j < end; j += THREADS * V) {
        const bool whole = j >= skew && j + V <= n;
        float z[V];
        if (whole) {
            const typename P::Vec v = *reinterpret_cast<const typename P::Loose *>(l + j);
#pragma unroll
            for (int k = 0; k < V; ++k) z[k] = to_f32(v[k]);
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k) z[k] = j + k >= skew && j + k < n ? to_f32(l[j + k]) : 0.0f;
        }
        if (counts) {
            unsigned w[V], any = 0;
#pragma unroll
            for (int k = 0; k < V; k += 4) {
                const uint4 four = *reinterpret_cast<const uint4 *>(words + (j - begin) + k);
                w[k] = four.x; w[k + 1] = four.y; w[k + 2] = four.z; w[k + 3] = four.w;
                any |= four.x | four.y | four.z | four.w;
            }
            if (any)
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (w[k] && j + k >= skew && j + k < n) z[k] = edit(z[k], w[k], j + k);
        }
        if (allowed) {
            const unsigned bits = bits_of(j);
#pragma unroll
            for (int k = 0; k < V; ++k) z[k] = bits >> k & 1 ? z[k] : -kInf;
        }
        if (whole) {
            typename P::Vec v;
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = from_f32<E>(z[k]);
            *reinterpret_cast<typename P::Loose *>(out + j) = v;
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (j + k >= skew && j + k < n) out[j + k] = from_f32<E>(z[k]);
        }
    }
}

}  // namespace
}  // namespace marl

using namespace marl;

extern "C" {

int marl_penalize(int32_t dtype, int32_t R, int32_t V, const void *logits, int64_t ld, int32_t L, const int32_t *history,
                  int64_t ld_history, const int32_t *length, const int32_t *prompt, const float *repetition, const float *presence,
                  const float *frequency, int32_t M, const int32_t *bias_id, const float *bias_value, const int32_t *allowed,
                  int64_t ld_allowed, void *out, int64_t ld_out, void *hip_stream)
{
    if (!known_dtype(dtype)) return MARL_ERR_BAD_DTYPE;
    if (R < 0 || R >= (1 << 24) || V < 1 || V >= (1 << 30) || ld < V || ld_out < V || L < 0 || L >= (1 << 24) || M < 0 || M > kMostBiases)
        return MARL_ERR_BAD_DIM;
    const int64_t bit_words = ((int64_t)V + 31) / 32;
    if ((history && L > 0 && ld_history < L) || (allowed && ld_allowed != 0 && ld_allowed < bit_words)) return MARL_ERR_BAD_DIM;
    if (logits && out == logits && ld_out != ld) return MARL_ERR_BAD_ARG;
    if (R == 0) return MARL_OK;
    if (!logits || !out || (L > 0 && !history) || (M > 0 && (!bias_id || !bias_value))) return MARL_ERR_NULL;
    PenalizeArgs p{};
    p.R = R; p.V = V; p.L = L; p.M = M;
    p.logits = logits; p.ld = ld; p.history = history; p.ld_history = ld_history; p.length = length; p.prompt = prompt;
    p.repetition = repetition; p.presence = presence; p.frequency = frequency; p.bias_id = bias_id; p.bias_value = bias_value;
    p.allowed = reinterpret_cast<const uint32_t *>(allowed); p.ld_allowed = ld_allowed; p.out = out; p.ld_out = ld_out;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return with_dtype(dtype, [&](auto e) {
        // pieces are counted from the line that the row's result begins in: up to 127 bytes before it
        constexpr int kSmall = 1024, kLarge = 8192;
        const bool small = V <= kSmall - 64;
        const int piece = small ? kSmall : kLarge;
        p.pieces = (int)(((int64_t)V + 63 + piece - 1) / piece);
        if ((int64_t)R * p.pieces >= ((int64_t)1 << 31)) return (int)MARL_ERR_BAD_DIM;
        const dim3 grid((unsigned)((int64_t)R * p.pieces));
        if (small) hipLaunchKernelGGL((penalize_kernel<decltype(e), 64, kSmall>), grid, dim3(64), 0, stream, p);
        else hipLaunchKernelGGL((penalize_kernel<decltype(e), 512, kLarge>), grid, dim3(512), 0, stream, p);
        return launched("penalize");
    });
}

}  // extern "C"
