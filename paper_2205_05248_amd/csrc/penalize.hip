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

// A place's word: how often it was generated (L < 2^24), which bias it has, whether it has one, whether it stood in the prompt.
constexpr unsigned kPrompt = 0x80000000u, kBiased = 0x40000000u, kCount = 0x00ffffffu;
constexpr int kBiasShift = 24, kNumbered = 64;         // with more biases than that in a piece a place looks for its own

// The biases of a piece, in their order; where they are numbered, that of a place's first entry is the sum of all of its entries.
struct BiasList {
    int *n, *at;
    float *value;                                      // [M] each
};

// The loads of the piece's logits, bits, first tokens and biases go out first; the history is counted while they are on their way.
template <typename E, int THREADS, int PIECE>
__global__ __launch_bounds__(THREADS) void penalize_kernel(PenalizeArgs p)
{
    typedef Piece<E> P;
    constexpr int V = P::V, kVectors = PIECE / THREADS / V, kBatch = 4;
    typedef int Tokens __attribute__((ext_vector_type(4)));
    typedef Tokens LooseTokens __attribute__((aligned(4)));
    extern __shared__ __attribute__((aligned(16))) char lds[];
    unsigned *words = reinterpret_cast<unsigned *>(lds);
    int *lists_at = reinterpret_cast<int *>(words + PIECE);
    const BiasList biases{lists_at, lists_at + 1, reinterpret_cast<float *>(lists_at + 1 + p.M)};
    const int64_t row = blockIdx.x / p.pieces;
    const int piece = blockIdx.x % p.pieces, lane = threadIdx.x % kWave;
    const E *l = static_cast<const E *>(p.logits) + row * p.ld;
    E *out = static_cast<E *>(p.out) + row * p.ld_out;
    const int skew = skew_of(out);                                     // entry j of the row is skew + j
    const int n = p.V + skew, begin = piece * PIECE, end = min(begin + PIECE, n);
    const int own = begin + (int)threadIdx.x * V;                      // vector q of the thread begins q THREADS V behind
    l -= skew;
    out -= skew;
    typename P::Vec z_raw[kVectors];
#pragma unroll
    for (int q = 0; q < kVectors; ++q) {
        const int j = own + q * THREADS * V;
        if (j >= skew && j + V <= n) {
            z_raw[q] = *reinterpret_cast<const typename P::Loose *>(l + j);
        } else if (j < end) {
#pragma unroll
            for (int k = 0; k < V; ++k) z_raw[q][k] = j + k >= skew && j + k < n ? l[j + k] : (E)0.0f;
        }
    }
    unsigned bits[kVectors];
    if (p.allowed) {
        typedef uint64_t LooseWord __attribute__((aligned(4)));
        const uint32_t *allowed = p.allowed + row * p.ld_allowed;
        const int last = (p.V - 1) / 32;
#pragma unroll
        for (int q = 0; q < kVectors; ++q) {
            const int e = own + q * THREADS * V - skew, low = min(max(e, 0), p.V - 1), word = min(low / 32, max(last - 1, 0));
            const uint64_t two = last > 0 ? *reinterpret_cast<const LooseWord *>(allowed + word) : allowed[0];
            bits[q] = (unsigned)(two >> (low - word * 32));
            if (e < 0) bits[q] <<= min(-e, 31);                        // (before the row nothing is written)
        }
    }
    // the first tokens and biases too, whatever the row's length is
    Tokens first[kBatch];
    auto tokens_at = [&](Tokens &to, int t, int most) {
        const int32_t *history = p.history + row * p.ld_history;
        if (t + 4 <= most) {
            to = *reinterpret_cast<const LooseTokens *>(history + t);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) to[k] = t + k < most ? history[t + k] : -1;
        }
    };
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
        if (q * THREADS * 4 < p.L) tokens_at(first[q], (q * THREADS + (int)threadIdx.x) * 4, p.L);
    const bool lists = threadIdx.x >= THREADS - kWave;                 // the last wave, which has the fewest tokens
    int bias_id = -1;
    float bias_value = 0.0f;
    if (lists && lane < p.M) {
        bias_id = p.bias_id[row * p.M + lane];
        bias_value = p.bias_value[row * p.M + lane];
    }
    const int length = p.length ? min(max(p.length[row], 0), p.L) : p.L;
    const int prompt = p.prompt ? min(max(p.prompt[row], 0), length) : 0;
    const float rho = p.repetition ? p.repetition[row] : 1.0f, presence = p.presence ? p.presence[row] : 0.0f;
    const float frequency = p.frequency ? p.frequency[row] : 0.0f;
    const bool counts = length > 0 || p.M > 0;
    if (counts) {
        // up to the end of the last vector, all of whose words are looked at
        for (int w = threadIdx.x * 4; w < (end - begin + V - 1) / V * V; w += THREADS * 4) *reinterpret_cast<uint4 *>(words + w) = make_uint4(0, 0, 0, 0);
        __syncthreads();
        const int before = skew - begin;                               // place of an id in the piece, if it has one
        auto place_of = [&](int id) {
            const int at = id + before;
            return id >= 0 && id < p.V && at >= 0 && at < end - begin ? at : -1;
        };
        if (lists && p.M > 0) {
            int m = 0;
            for (int base = 0; base < p.M; base += kWave) {            // one wave keeps the order
                if (base > 0) {
                    bias_id = base + lane < p.M ? p.bias_id[row * p.M + base + lane] : -1;
                    bias_value = base + lane < p.M ? p.bias_value[row * p.M + base + lane] : 0.0f;
                }
                const int at = place_of(bias_id);
                const unsigned long long all = __ballot(at >= 0);
                if (at >= 0) {
                    const int to = m + __popcll(all & ((1ull << lane) - 1));
                    biases.at[to] = at;
                    biases.value[to] = bias_value;
                }
                m += __popcll(all);
            }
            if (lane == 0) *biases.n = m;
            wave_sync();
            if (m <= kNumbered) {
                const int at = lane < m ? biases.at[lane] : -1;
                float sum = 0.0f;
                bool leads = lane < m;
                for (int k = 0; k < m; ++k) {
                    const bool same = biases.at[k] == at;
                    sum += same ? biases.value[k] : 0.0f;
                    leads = leads && !(same && k < lane);
                }
                wave_sync();
                if (leads) {
                    biases.value[lane] = sum;
                    atomicOr(&words[at], kBiased | (unsigned)lane << kBiasShift);
                }
            } else {
                for (int k = lane; k < m; k += kWave) atomicOr(&words[biases.at[k]], kBiased);
            }
        }
        for (int base = 0; base < length; base += THREADS * 4 * kBatch) {
            if (base > 0)
#pragma unroll
                for (int q = 0; q < kBatch; ++q) tokens_at(first[q], base + (q * THREADS + (int)threadIdx.x) * 4, length);
#pragma unroll
            for (int q = 0; q < kBatch; ++q)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int t = base + (q * THREADS + (int)threadIdx.x) * 4 + k, at = place_of(first[q][k]);
                    if (t < length && at >= 0) {
                        if (t >= prompt) atomicAdd(&words[at], 1u);
                        else atomicOr(&words[at], kPrompt);
                    }
                }
        }
        __syncthreads();
    }
    const float inverse = 1.0f / rho;
    const bool divides = !(rho >= 1e-6f && rho <= 1e6f);               // the reciprocal or its products may leave the range of fp32
#pragma unroll
    for (int q = 0; q < kVectors; ++q) {
        const int j = own + q * THREADS * V;
        if (j >= end) continue;
        float z[V];
#pragma unroll
        for (int k = 0; k < V; ++k) z[k] = to_f32(z_raw[q][k]);
        if (counts) {
            unsigned w[V], any = 0;
#pragma unroll
            for (int k = 0; k < V; k += 4) {
                const uint4 four = *reinterpret_cast<const uint4 *>(words + (j - begin) + k);
                w[k] = four.x; w[k + 1] = four.y; w[k + 2] = four.z; w[k + 3] = four.w;
                any |= four.x | four.y | four.z | four.w;
            }
            if (any) {
                float less[V];
                if (divides) {
#pragma unroll
                    for (int k = 0; k < V; ++k) less[k] = z[k] > 0.0f ? z[k] / rho : z[k] * rho;
                } else {
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        // z / rho from its reciprocal, corrected by what is left over: as near as a division, which is four times as long
                        const float guess = z[k] * inverse, divided = fmaf(fmaf(-guess, rho, z[k]), inverse, guess);
                        const bool usual = fabsf(z[k]) < 1e30f && fabsf(z[k]) > 1e-30f;
                        less[k] = z[k] > 0.0f ? (usual ? divided : guess) : z[k] * rho;
                    }
                }
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const unsigned c = w[k] & kCount;
                    const float seen = w[k] & (kPrompt | kCount) ? less[k] : z[k];
                    z[k] = c ? (seen - presence) - frequency * (float)c : seen;
                }
                if (any & kBiased)
#pragma unroll
                    for (int k = 0; k < V; ++k)
                        if (w[k] & kBiased) {
                            if (*biases.n <= kNumbered) z[k] += biases.value[w[k] >> kBiasShift & (kNumbered - 1)];
                            else {
                                float sum = 0.0f;
                                for (int m = 0; m < *biases.n; ++m) sum += biases.at[m] == j - begin + k ? biases.value[m] : 0.0f;
                                z[k] += sum;
                            }
                        }
            }
        }
        if (p.allowed)
#pragma unroll
            for (int k = 0; k < V; ++k) z[k] = bits[q] >> k & 1 ? z[k] : -kInf;
        typename P::Vec v;
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = from_f32<E>(z[k]);
        if (j >= skew && j + V <= n) {
            __builtin_nontemporal_store(v, reinterpret_cast<typename P::Loose *>(out + j));
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (j + k >= skew && j + k < n) out[j + k] = v[k];
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
        // Pieces are counted from the line that the row's result begins in: up to 127 bytes before it.  Every piece reads the history, but with
        // four of 8192 places on a compute unit some pass logits while others count: 777 rows of 50021 in fp16 with 4096 tokens on
        // average, 64 biases and a mask take 61 us (24 without any of them, a copy 22: reading the tokens and looking for their places in every piece
        // takes 15 of the rest, counting them and the edit of what they touch 7, listing the biases, by one wave before the pass, 7 to 15; 65 with
        // stores through the caches), with pieces of 16384 and 1024 threads 82, with 4096 and 256 threads 64.  Rows of one wave up to 960: 24 x 40 with 120 tokens take 6.4 us, most of it the launch.
        const auto go = [&](auto kernel, int threads, int piece) {
            const size_t lds = piece * sizeof(unsigned) + (1 + 2 * (size_t)M) * sizeof(int);       // 40 KB at most
            p.pieces = (int)(((int64_t)V + 63 + piece - 1) / piece);
            if (!fits_a_launch((int64_t)R * p.pieces, threads)) return (int)MARL_ERR_BAD_DIM;
            hipLaunchKernelGGL(kernel, dim3((unsigned)((int64_t)R * p.pieces)), dim3(threads), lds, stream, p);
            return launched("penalize");
        };
        if (V <= 1024 - 64) return go(penalize_kernel<decltype(e), 64, 1024>, 64, 1024);
        return go(penalize_kernel<decltype(e), 512, 8192>, 512, 8192);
    });
}

}  // extern "C"
