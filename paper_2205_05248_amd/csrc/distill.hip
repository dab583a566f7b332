// Divergence of a student's logits from a teacher's kept alternatives, and the logits' gradient.  The alternatives' places are left out of
// the sum over the row and added at the end, so that the probability of all others is a sum of its own and not one minus a number next to
// one.  Forward and backward are bound by the bytes of the logits where rows are long: 8191 x 50021 fp16 with 20 alternatives 205 us forward (4.0
// TB/s) and 321 backward (5.1 TB/s).  Short rows by their instructions: 409600 x 40 fp32 with a mask and five alternatives 41 and 42 us (2.0 and 3.5
// TB/s).  Few rows by the chain of loads and sums: 16 x 131072 bf16 with 50 alternatives 5 us, and 7.8 of a wave a row that joins the parts.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "logit_rows.h"

namespace marl {
namespace {

constexpr int kMostKept = 64;                          // a lane of a wave each

struct DistillArgs : LogitRows {
    int K, tail;
    const int32_t *top_id;
    const float *top_value;
    float *loss, *log_sum, *log_rest;
    // gradient
    const float *in_log_sum, *in_log_rest, *grad_loss;
    void *grad_logits;
    int64_t ld_grad;
    // long rows in parts
    int parts, per;                    // parts of a row, chunks of a part
    float *stats;                      // [R, parts, 2]
};

// sum e^(z - m) over a set, m its maximum; m = -inf is the empty set.
struct Sum { float m, s; };

// Between two empty sets, or behind a maximum of NaN, the distance is NaN and counts as far; a maximum keeps NaN.
__device__ __forceinline__ float far_exp(float v) { return exp_of(fmaxf(v, -1e30f)); }
__device__ __forceinline__ Sum join(Sum a, Sum b)
{
    const float M = max_nan(a.m, b.m);
    return {M, a.s * far_exp(a.m - M) + b.s * far_exp(b.m - M)};
}
__device__ __forceinline__ Sum join_wave(Sum v)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) v = join(v, {__shfl_xor(v.m, d), __shfl_xor(v.s, d)});
    return v;
}
__device__ __forceinline__ float add(float a, float b) { return a + b; }
template <int LANES, int D = 1>
__device__ __forceinline__ double sum_lanes(double v)
{
    if constexpr (D < LANES) {
        const uint64_t bits = __builtin_bit_cast(uint64_t, v);
        const unsigned low = __float_as_uint(across<D>(__uint_as_float((unsigned)bits))), high = __float_as_uint(across<D>(__uint_as_float((unsigned)(bits >> 32))));
        return sum_lanes<LANES, 2 * D>(v + __builtin_bit_cast(double, (uint64_t)high << 32 | low));
    } else {
        return v;
    }
}

// What the two sums of a row give: of the kept places and of all others.
struct RowSums {
    float M, log_s, log_rest;
    bool none, bad, some_left;
};
__device__ __forceinline__ RowSums row_sums(Sum kept, Sum rest)
{
    RowSums r;
    const Sum all = join(kept, rest);
    r.M = all.m;
    r.none = all.m == -kInf;
    r.bad = !(all.m < kInf);
    r.some_left = !(rest.m == -kInf);
    r.log_s = logf(all.s);
    // next to 1 from what is taken away, which is small; else from the sum itself
    const float taken = kept.s * far_exp(kept.m - all.m);
    r.log_rest = 2.0f * taken < all.s ? log1pf(-taken / all.s) : (rest.m - all.m) + (logf(rest.s) - r.log_s);
    if (!r.some_left) r.log_rest = -kInf;
    return r;
}

// An alternative as a lane holds it.
struct Kept { int id; float value, z, logit; bool is; };
// listed_at: what is listed, asked for before the row is there; kept_of: what the row, which may be in shared memory, says to it.
__device__ __forceinline__ Kept listed_at(const DistillArgs &p, int64_t row, int k)
{
    Kept a{-1, -kInf, -kInf, -kInf, false};
    if (k < p.K) {
        a.id = p.top_id[row * p.K + k];
        a.value = p.top_value[row * p.K + k];
    }
    return a;
}
template <typename E>
__device__ __forceinline__ void kept_of(const DistillArgs &p, Kept &a, const E *l, const uint8_t *av)
{
    const bool in = a.id >= 0 && a.id < p.V;
    a.id = in ? a.id : -1;
    const bool available = in && (!av || av[a.id]);
    a.logit = available ? to_f32(l[a.id]) : -kInf;
    a.is = available && !(a.logit < p.lowest);
    a.value = !a.is ? -kInf : a.value == kInf ? __builtin_nanf("") : a.value;
    a.z = a.is ? rounded(p.scale, a.logit) : -kInf;
}
template <typename E>
__device__ __forceinline__ Kept kept_at(const DistillArgs &p, const E *l, const uint8_t *av, int64_t row, int k)
{
    Kept a = listed_at(p, row, k);
    kept_of(p, a, l, av);
    return a;
}

// The teacher's side: log p of a value is value - top - log_total, p its exponential.
struct Teacher { float top, total, log_total; };
// A constant in scalar registers where it is used: in vector registers, kept through the kernel, the twelve below leave room for five waves in place of seven on
// rows of 1000 (50000 rows bf16, 20 alternatives: 100 -> 122 us).
__device__ __forceinline__ double kept_scalar(double v)
{
    asm volatile("" : "+s"(v));
    return v;
}
// p of an alternative whose value is its log probability, in 64 bits: what the teacher has for all other places is one minus the sum of these, of a sure teacher a
// small number, for which its log probabilities have the digits and their exponentials in fp32 do not (of 1e-6 a twentieth was lost, of 2e-8 all).  e^v = 2^n e^r
// with |r| <= log(2) / 2, whose series ends at r^11: the rest is below 2^-46.  (Half as long as the library's exponential, which needs no bounds; what is below them is 0 in
// fp32, and above them infinite.)
__device__ __forceinline__ double exact_part(const Kept &a)
{
    const float v = __builtin_elementwise_minimum(max_nan(a.value, -150.0f), 100.0f), n = __builtin_rintf(kLog2e * v);              // NaN stays
    const double r = fma(-(double)n, 0.69314718055994530942, (double)v);
    const double rr = r * r;
    double factorial = 39916800, odd = 1 / factorial, even = 11 / factorial;       // 11!; two sums, neither waits for the other
#pragma unroll
    for (int i = 9; i > 0; i -= 2) {
        factorial /= (i + 1) * (i + 2);
        odd = fma(odd, rr, kept_scalar(1 / factorial));
        even = fma(even, rr, kept_scalar(i / factorial));
    }
    return a.is ? __builtin_ldexp(fma(odd, r, even), (int)n) : 0.0;
}
__device__ __forceinline__ float left_of(double sum) { return sum >= 1.0 ? 0.0f : (float)(1.0 - sum); }                // NaN stays
// The same of values that are any logits.
__device__ __forceinline__ float share(const Teacher &t, const Kept &a)
{
    return !a.is ? 0.0f : t.total > 0.0f ? expf(a.value - t.top) / t.total : t.total == 0.0f ? 0.0f : __builtin_nanf("");
}
__device__ __forceinline__ float probability(const Teacher &t, int tail, const Kept &a) { return !tail ? share(t, a) : a.is ? expf(a.value) : 0.0f; }
// p (log p - log q), 0 where p is.
__device__ __forceinline__ float part_of_loss(float p, float log_p, float log_q) { return p == 0.0f ? 0.0f : p * (log_p - log_q); }
__device__ __forceinline__ void put_row(const DistillArgs &p, int64_t row, const RowSums &r, float loss, float left)
{
    const float nan = __builtin_nanf("");
    if (p.tail && r.some_left) loss += part_of_loss(left, logf(left), r.log_rest);
    p.loss[row] = r.bad ? nan : r.none ? 0.0f : loss;
    if (p.log_sum) p.log_sum[row] = r.bad ? nan : r.none ? -kInf : r.M + r.log_s;
    if (p.tail && p.log_rest) p.log_rest[row] = r.bad ? nan : r.log_rest;
}

// The same index at a lower lane.
__device__ __forceinline__ bool met_before(int id, int K)
{
    const int lane = threadIdx.x % kWave;
    bool met = false;
    for (int k = 0; k < K; ++k) met = met || (k < lane && __builtin_amdgcn_readlane(id, k) == id);
    return met;
}

__device__ __forceinline__ Teacher teacher_of(const Kept &a)
{
    Teacher t;
    t.top = all_lanes<kWave>(a.is ? a.value : -kInf, max_nan);
    t.total = all_lanes<kWave>(a.is && a.value != -kInf ? expf(a.value - t.top) : 0.0f, add);
    t.log_total = logf(t.total);
    return t;
}

// A wave finishes a row from the sum over the places that are not listed and the alternatives that its lanes hold.
__device__ __forceinline__ void finish_row(const DistillArgs &p, int64_t row, Sum rest, const Kept &a)
{
    const bool met = met_before(a.id, p.K);            // (in all lanes: it reads them)
    Sum kept;
    kept.m = all_lanes<kWave>(a.z, max_nan);
    kept.s = all_lanes<kWave>(a.is && !met ? exp_of(a.z - kept.m) : 0.0f, add);
    const RowSums r = row_sums(kept, rest);
    const Teacher t = teacher_of(a);
    const double part = p.tail ? exact_part(a) : 0.0;
    const float prob = p.tail ? (float)part : share(t, a);
    const float log_p = p.tail ? a.value : (a.value - t.top) - t.log_total;
    const float loss = all_lanes<kWave>(part_of_loss(prob, log_p, (a.z - r.M) - r.log_s), add);
    const float left = p.tail ? left_of(sum_lanes<kWave>(part)) : 0.0f;
    if (threadIdx.x % kWave == 0) put_row(p, row, r, loss, left);
}

// ---------------------------------------------------------------------------------- long rows
constexpr int kHeld = 32;                              // logits of a lane at a time
constexpr int kChunk = kThreads * kHeld;               // of a workgroup
constexpr int kMostChunks = 16;                        // of a part: its places have a bit each in shared memory

// The listed places of a part of a row as bits, counted from `begin`.
struct Listed {
    unsigned bits[kMostChunks * kChunk / 32];
    // id: the thread's alternative; the row begins `skew` behind where places are counted from
    __device__ __forceinline__ void mark(const DistillArgs &p, int id, int skew, int64_t begin, int64_t end)
    {
        const int words = (int)((end - begin + 31) / 32);
        for (int w = threadIdx.x; w < words; w += kThreads) bits[w] = 0;
        __syncthreads();
        if ((int)threadIdx.x < p.K) {
            const int64_t at = id + (int64_t)skew - begin;
            if (id >= 0 && id < p.V && at >= 0 && at < end - begin) atomicOr(&bits[at / 32], 1u << (at % 32));
        }
        __syncthreads();
    }
    // of V places from `at` on, a multiple of V
    template <int V>
    __device__ __forceinline__ unsigned of(int at) const { return bits[at / 32] >> (at % 32) & ((1u << V) - 1); }
};

template <int N>
__device__ __forceinline__ void take(Sum &st, const float (&l)[N], float scale)
{
    float top = l[0];
#pragma unroll
    for (int k = 1; k < N; ++k) top = max_nan(top, l[k]);
    const float M = max_nan(st.m, top == -kInf ? -kInf : rounded(scale, top));
    if (!(M == st.m)) st = {M, st.s * far_exp(st.m - M)};
#pragma unroll
    for (int k = 0; k < N; ++k) st.s += far_exp(rounded(scale, l[k]) - M);
}

template <typename E>
__global__ __launch_bounds__(kThreads, 8) void long_rows_kernel(DistillArgs p)
{
    constexpr int V = Piece<E>::V;
    __shared__ Listed listed;
    __shared__ Sum part[kThreads / kWave];
    const int64_t row = blockIdx.x / p.parts;
    const int piece = blockIdx.x % p.parts;
    const E *l = static_cast<const E *>(p.logits) + row * p.ld;
    const uint8_t *av = p.avail ? p.avail + row * p.ld_avail : nullptr;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int skew = skew_of(l), n = p.V + skew;                       // entry j of the row is skew + j
    l -= skew;
    if (av) av -= skew;
    const int64_t begin = (int64_t)piece * p.per * kChunk, end = piece + 1 < p.parts ? begin + (int64_t)p.per * kChunk : n;
    listed.mark(p, listed_at(p, row, threadIdx.x).id, skew, begin, end);
    Sum st{-kInf, 0.0f};
    int64_t base = begin;
    for (; base + kChunk <= end; base += kChunk) {
        float held[kHeld];
        unsigned out = 0;
#pragma unroll
        for (int q = 0; q < kHeld / V; ++q) {
            const int j = (int)base + (q * kThreads + (int)threadIdx.x) * V;
            read_piece<E>(l, av, j, skew, n, held + q * V);
            out |= listed.of<V>(j - (int)begin) << (q * V);
        }
        if (out)                                       // (once for all pieces: a branch between their loads would wait for each)
#pragma unroll
            for (int k = 0; k < kHeld; ++k) held[k] = out >> k & 1 ? -kInf : held[k];
        take(st, held, p.scale);
    }
    for (; base + wave * (kWave * V) < end; base += kThreads * V) {    // what is left: a piece at a time, and no more than there are
        float some[V];
        const int j = (int)base + (int)threadIdx.x * V;
        read_piece<E>(l, av, j, skew, n, some);
        const unsigned out = j < end ? listed.of<V>(j - (int)begin) : 0;
        if (out)
#pragma unroll
            for (int k = 0; k < V; ++k) some[k] = out >> k & 1 ? -kInf : some[k];
        take(st, some, p.scale);
    }
    st = join_wave(st);
    if (lane == 0) part[wave] = st;
    __syncthreads();
    if (wave != 0) return;
    st = part[0];
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) st = join(st, part[w]);
    if (p.parts > 1) {
        if (lane == 0) {
            float *to = p.stats + (row * p.parts + piece) * 2;
            to[0] = st.m; to[1] = st.s;
        }
    } else {
        finish_row(p, row, st, kept_at(p, l + skew, av ? av + skew : nullptr, row, lane));
    }
}

// A wave per row joins its parts.
template <typename E>
__global__ __launch_bounds__(kWave) void join_kernel(DistillArgs p)
{
    const int64_t row = blockIdx.x;
    const Kept mine = kept_at(p, static_cast<const E *>(p.logits) + row * p.ld, p.avail ? p.avail + row * p.ld_avail : nullptr, row, threadIdx.x);
    Sum st{-kInf, 0.0f};
    for (int k = threadIdx.x; k < p.parts; k += kWave) {
        const float *from = p.stats + (row * p.parts + k) * 2;
        st = join(st, {from[0], from[1]});
    }
    finish_row(p, row, join_wave(st), mine);
}

// What the gradient of a row needs: places that are not kept get C e^(z - base), kept ones W e^(z - log_sum) - p, all times `by`.
struct RowGrad { float log_sum, base, W, C, by; };
__device__ __forceinline__ RowGrad row_grad(const DistillArgs &p, int64_t row, float sum, float left)
{
    RowGrad g;
    g.log_sum = p.in_log_sum[row];
    g.by = p.scale * p.grad_loss[row];
    if (p.grad_loss[row] == 0.0f) g.by = 0.0f;
    const float log_rest = p.tail ? p.in_log_rest[row] : 0.0f;
    if (log_rest == -kInf) left = 0.0f;
    g.W = sum + left;
    // (W - left / q_r) q = (W q_r - left) (q / q_r): the quotient of two small numbers is formed in the exponent
    g.C = p.tail ? g.W * exp_of(log_rest) - left : g.W;
    g.base = g.log_sum + log_rest;
    return g;
}
// factor * e^v as the square of a root, which the hardware exponential does not flush where e^v is subnormal
__device__ __forceinline__ float times_exp(float factor, float v)
{
    const float root = __builtin_amdgcn_exp2f(0.5f * kLog2e * max_nan(v, -200.0f));
    return root * (root * factor);
}
__device__ __forceinline__ float other_grad(const RowGrad &g, float logit, float scale, float lowest)
{
    return logit < lowest || g.by == 0.0f ? 0.0f : g.by * times_exp(g.C, rounded(scale, logit) - g.base);
}
__device__ __forceinline__ float kept_grad(const RowGrad &g, float logit, float prob, float scale, float lowest)
{
    return logit < lowest || g.by == 0.0f ? 0.0f : g.by * (times_exp(g.W, rounded(scale, logit) - g.log_sum) - prob);
}

// A workgroup takes `per` chunks of a row (the whole row if it overwrites the logits: the kept ones are looked at before any is gone).
template <typename E>
__global__ __launch_bounds__(kThreads) void long_grad_kernel(DistillArgs p)
{
    typedef Piece<E> P;
    constexpr int V = P::V, kPieces = 4, kStep = kThreads * V * kPieces;
    __shared__ Listed listed;
    __shared__ int ids[kMostKept];
    __shared__ float probs[kMostKept], total, left;
    const int64_t row = blockIdx.x / p.parts;
    const int piece = blockIdx.x % p.parts;
    const E *l = static_cast<const E *>(p.logits) + row * p.ld;
    const uint8_t *av = p.avail ? p.avail + row * p.ld_avail : nullptr;
    E *out = static_cast<E *>(p.grad_logits) + row * p.ld_grad;
    const Kept a = kept_at(p, l, av, row, threadIdx.x);
    if (threadIdx.x < kWave) {
        const Teacher t = teacher_of(a);
        const double part = p.tail ? exact_part(a) : 0.0, parts = p.tail ? sum_lanes<kWave>(part) : 0.0;
        const float prob = p.tail ? (float)part : share(t, a), sum = p.tail ? (float)parts : all_lanes<kWave>(prob, add);
        ids[threadIdx.x] = a.is ? a.id : -1;
        probs[threadIdx.x] = prob;
        if (threadIdx.x == 0) total = sum, left = p.tail ? left_of(parts) : 0.0f;
    }
    const int skew = skew_of(l), n = p.V + skew;                       // entry j of the row is skew + j
    const int64_t span = (int64_t)p.per * kStep;
    l -= skew;
    out -= skew;
    if (av) av -= skew;
    const int64_t stop = piece + 1 < p.parts ? (int64_t)(piece + 1) * span : n;
    for (int64_t from = (int64_t)piece * span; from < stop; from += kMostChunks * kChunk) {
        const int64_t to = from + kMostChunks * kChunk < stop ? from + kMostChunks * kChunk : stop;
        __syncthreads();
        listed.mark(p, a.id, skew, from, to);
        const RowGrad g = row_grad(p, row, total, left);
        auto put = [&](const float *held, int j) {
            typename P::Vec v;
            const unsigned marked = listed.of<V>(j - (int)from);
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = from_f32<E>(other_grad(g, held[k], p.scale, p.lowest));
            if (marked)
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (marked >> k & 1) {
                        float prob = 0.0f;
                        for (int c = 0; c < p.K; ++c) prob += ids[c] == j + k - skew ? probs[c] : 0.0f;
                        v[k] = from_f32<E>(kept_grad(g, held[k], prob, p.scale, p.lowest));
                    }
            if (j >= skew && j + V <= n) {
                *reinterpret_cast<typename P::Loose *>(out + j) = v;
            } else {
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (j + k >= skew && j + k < n) out[j + k] = v[k];
            }
        };
        int64_t base = from;
        for (; base + kStep <= to; base += kStep) {
            float held[kPieces][V];
#pragma unroll
            for (int q = 0; q < kPieces; ++q) read_piece<E>(l, av, (int)base + (q * kThreads + (int)threadIdx.x) * V, skew, n, held[q]);
#pragma unroll
            for (int q = 0; q < kPieces; ++q) put(held[q], (int)base + (q * kThreads + (int)threadIdx.x) * V);
        }
        for (; base + (threadIdx.x / kWave) * (kWave * V) < to; base += kThreads * V) {                    // what is left: a piece at a time
            float held[V];
            const int j = (int)base + (int)threadIdx.x * V;
            if (j >= to) continue;
            read_piece<E>(l, av, j, skew, n, held);
            put(held, j);
        }
    }
}

// ---------------------------------------------------------------------------------- short rows
// G lanes hold a row of at most G N logits; lane `sub` of them looks at alternatives sub, sub + G, ..., of which the first stays with it.
template <int G>
struct ShortTeacher {
    Teacher t;
    float sum, left, first;                            // of all alternatives, of all other places, of the lane's first alternative
    unsigned marked;                                   // of the lane's own entries j G + sub, bit j
};
template <typename E, int G>
__device__ __forceinline__ ShortTeacher<G> short_teacher(const DistillArgs &p, Kept &first, const E *l, const uint8_t *av, int64_t row, bool there)
{
    const int lane = threadIdx.x % kWave, sub = lane % G;
    ShortTeacher<G> s{{-kInf, 0.0f, 0.0f}, 0.0f, 0.0f, 0.0f, 0};
    double sum = 0.0;
    if (!there) first.id = -1;
    kept_of(p, first, l, av);
    Kept a = first;
    for (int base = 0;;) {
        for (int k = 0; k < G && base + k < p.K; ++k) {
            const int id = __shfl(a.id, lane - sub + k);
            s.marked |= id >= 0 && id % G == sub ? 1u << (id / G) : 0u;
        }
        if (p.tail) {
            const double part = exact_part(a);
            if (base == 0) s.first = (float)part;
            sum += part;
        } else {
            const float top = max_nan(s.t.top, a.value);
            if (!(top == s.t.top)) s.t.total *= s.t.top == -kInf ? 0.0f : expf(s.t.top - top);
            s.t.top = top;
            s.t.total += a.is && a.value != -kInf ? expf(a.value - top) : 0.0f;
        }
        if ((base += G) >= p.K) break;
        a = there ? kept_at(p, l, av, row, base + sub) : Kept{-1, -kInf, -kInf, -kInf, false};
    }
    if (p.tail) {
        sum = sum_lanes<G>(sum);
        s.sum = (float)sum;
        s.left = left_of(sum);
    } else {
        const float top = all_lanes<G>(s.t.top, max_nan);
        s.t.total = all_lanes<G>(s.t.top == -kInf ? 0.0f : s.t.total * expf(s.t.top - top), add);
        s.t.top = top;
        s.t.log_total = logf(s.t.total);
        s.sum = s.t.total == 0.0f ? 0.0f : s.t.total > 0.0f ? 1.0f : __builtin_nanf("");
        s.first = share(s.t, first);
    }
    return s;
}

// Where a row and its mask lie in the room that a wave's rows were brought to.
template <typename E, int G, int N>
__device__ __forceinline__ const E *row_in(const DistillArgs &p, const FlatRows<E, G, N> &rows, int64_t first, int64_t row)
{
    return rows.entries + (int)((reinterpret_cast<uintptr_t>(static_cast<const E *>(p.logits) + first * p.V) & 15) / sizeof(E)) + (int)(row - first) * p.V;
}
template <typename E, int G, int N>
__device__ __forceinline__ const uint8_t *mask_in(const DistillArgs &p, const FlatRows<E, G, N> &rows, int64_t first, int64_t row)
{
    return !p.avail || p.ld_avail == 0 ? p.avail : rows.mask + (int)(reinterpret_cast<uintptr_t>(p.avail + first * p.V) & 15) + (int)(row - first) * p.V;
}

template <typename E, int G, int N, bool FLAT>
__global__ __launch_bounds__(kThreads) void short_rows_kernel(DistillArgs p)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, sub = lane % G;
    const int64_t first = ((int64_t)blockIdx.x * (kThreads / kWave) + wave) * (kWave / G), row = first + lane / G;
    if (first >= p.R) return;                                          // the whole wave
    const bool there = row < p.R;
    const int64_t own = there ? row : first;
    const E *l = static_cast<const E *>(p.logits) + own * p.ld;
    const uint8_t *av = p.avail ? p.avail + own * p.ld_avail : nullptr;
    __shared__ __attribute__((aligned(16))) FlatRows<E, FLAT ? G : 1, FLAT ? N : 1> rows[FLAT ? kThreads / kWave : 1];
    Kept listed = listed_at(p, own, sub);
    float held[N];
    if constexpr (FLAT) {
        rows[wave].read(p, first, row, there, -1, held);
        l = row_in(p, rows[wave], first, own);
        av = mask_in(p, rows[wave], first, own);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int k = j * G + sub;
            held[j] = there && k < p.V && (!av || av[k]) ? to_f32(l[k]) : -kInf;
        }
    }
    const ShortTeacher<G> s = short_teacher<E, G>(p, listed, l, av, own, there);
    float top_in = -kInf, top_out = -kInf;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        top_in = max_nan(top_in, s.marked >> j & 1 ? held[j] : -kInf);
        top_out = max_nan(top_out, s.marked >> j & 1 ? -kInf : held[j]);
    }
    auto of_scale = [&](float v) { return v == -kInf ? v : rounded(p.scale, v); };
    Sum kept{of_scale(all_lanes<G>(top_in, max_nan)), 0.0f}, rest{of_scale(all_lanes<G>(top_out, max_nan)), 0.0f};
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const bool in = s.marked >> j & 1;
        const float e = far_exp(rounded(p.scale, held[j]) - (in ? kept.m : rest.m));
        kept.s += in ? e : 0.0f;
        rest.s += in ? 0.0f : e;
    }
    kept.s = all_lanes<G>(kept.m == -kInf ? 0.0f : kept.s, add);
    rest.s = all_lanes<G>(rest.m == -kInf ? 0.0f : rest.s, add);
    const RowSums r = row_sums(kept, rest);
    float loss = 0.0f;
    for (int base = 0; base < p.K; base += G) {
        const Kept a = base == 0 ? listed : there ? kept_at(p, l, av, own, base + sub) : Kept{-1, -kInf, -kInf, -kInf, false};
        const float prob = base == 0 ? s.first : probability(s.t, p.tail, a);
        loss += part_of_loss(prob, p.tail ? a.value : (a.value - s.t.top) - s.t.log_total, (a.z - r.M) - r.log_s);
    }
    loss = all_lanes<G>(loss, add);
    if (there && sub == 0) put_row(p, row, r, loss, s.left);
}

template <typename E, int G, int N, bool FLAT>
__global__ __launch_bounds__(kThreads) void short_grad_kernel(DistillArgs p)
{
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, sub = lane % G;
    const int64_t first = ((int64_t)blockIdx.x * (kThreads / kWave) + wave) * (kWave / G), row = first + lane / G;
    if (first >= p.R) return;                                          // the whole wave
    const bool there = row < p.R;
    const int64_t own = there ? row : first;
    const E *l = static_cast<const E *>(p.logits) + own * p.ld;
    const uint8_t *av = p.avail ? p.avail + own * p.ld_avail : nullptr;
    E *out = static_cast<E *>(p.grad_logits) + own * p.ld_grad;
    __shared__ __attribute__((aligned(16))) FlatRows<E, FLAT ? G : 1, FLAT ? N : 1> rows[FLAT ? kThreads / kWave : 1];
    Kept listed = listed_at(p, own, sub);
    float held[N];
    if constexpr (FLAT) {
        rows[wave].read(p, first, row, there, -1, held);
        l = row_in(p, rows[wave], first, own);
        av = mask_in(p, rows[wave], first, own);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int k = j * G + sub;
            held[j] = there && k < p.V && (!av || av[k]) ? to_f32(l[k]) : -kInf;
        }
    }
    const ShortTeacher<G> s = short_teacher<E, G>(p, listed, l, av, own, there);
    const RowGrad g = row_grad(p, own, s.sum, s.left);
    constexpr int kRounds = kMostKept / G;                             // the kept ones' logits are read before any is overwritten
    int ids[kRounds];
    float grads[kRounds];
    {                                                                  // listed twice: both parts
        const float prob = s.first;
        float sum = 0.0f;
        for (int k = 0; k < G && k < p.K; ++k) {
            const int id = __shfl(listed.id, lane - sub + k);
            const float part = __shfl(prob, lane - sub + k);
            sum += id == listed.id ? part : 0.0f;
        }
        ids[0] = listed.id;
        grads[0] = sum;
    }
#pragma unroll
    for (int c = 0; c < kRounds; ++c) {
        if (c > 0) ids[c] = -1;
        if (c * G >= p.K) continue;
        const Kept a = c == 0 ? listed : there ? kept_at(p, l, av, own, c * G + sub) : Kept{-1, -kInf, -kInf, -kInf, false};
        if (c > 0) ids[c] = a.id, grads[c] = 0.0f;
        if (p.K > G && a.is) {
            grads[c] = 0.0f;
            for (int k = 0; k < p.K; ++k)
                if (p.top_id[own * p.K + k] == a.id) {
                    const float value = p.top_value[own * p.K + k];
                    grads[c] += probability(s.t, p.tail, Kept{a.id, value == kInf ? __builtin_nanf("") : value, a.z, a.logit, true});
                }
        }
        grads[c] = a.is ? kept_grad(g, a.logit, grads[c], p.scale, p.lowest) : 0.0f;
    }
    wave_sync();                                                       // all of the row is read before any of it is overwritten
    E *to = out;
    int skew = 0;
    if constexpr (FLAT) {
        skew = (int)((reinterpret_cast<uintptr_t>(static_cast<E *>(p.grad_logits) + first * p.V) & 15) / sizeof(E));
        to = rows[wave].entries + skew + (int)(own - first) * p.V;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int k = j * G + sub;
        if (there && k < p.V && !(s.marked >> j & 1)) to[k] = from_f32<E>(other_grad(g, held[j], p.scale, p.lowest));
    }
#pragma unroll
    for (int c = 0; c < kRounds; ++c)
        if (c * G < p.K && there && ids[c] >= 0) to[ids[c]] = from_f32<E>(grads[c]);
    if constexpr (FLAT) {
        wave_sync();
        bring_back<E, kWave * N>(static_cast<E *>(p.grad_logits), first * p.V, (int)min((int64_t)(kWave / G), p.R - first) * p.V, skew, rows[wave].entries);
    }
}

// Rows up to this long are held by one wave or a part of it.
constexpr int kShort = 2048;

Cut part_cut(int R, int V)
{
    Cut cut = cut_of(R, V, kChunk, false);
    if (cut.per > kMostChunks) cut = {(cut.parts * cut.per + kMostChunks - 1) / kMostChunks, kMostChunks};
    // a row that begins behind a line may end in one chunk more than it has
    if ((int64_t)V + 127 > (int64_t)cut.parts * cut.per * kChunk) cut.parts += 1;
    return cut;
}

// A short row takes up to 64 lanes, a long one 256.
bool rows_fit(int R, int V) { return V > kShort ? R < 1 << 24 : R < 1 << 26; }

size_t distill_workspace(int R, int V)
{
    if (V <= kShort) return 0;
    const Cut cut = part_cut(R, V);
    return cut.parts == 1 ? 0 : ((size_t)R * cut.parts * 2 * sizeof(float) + 255) / 256 * 256;
}

template <typename E>
int run_forward(DistillArgs p, hipStream_t stream)
{
    if (p.V <= kShort) {
        auto go = [&](auto kernel, int G) {
            const int64_t rows = (int64_t)(kThreads / kWave) * (kWave / G);
            hipLaunchKernelGGL(kernel, dim3((unsigned)((p.R + rows - 1) / rows)), dim3(kThreads), 0, stream, p);
            return launched("distill");
        };
        if (rows_are_flat(p)) {
            if (p.V <= 16) return go(short_rows_kernel<E, 4, 4, true>, 4);
            if (p.V <= 48) return go(short_rows_kernel<E, 8, 6, true>, 8);
            if (p.V <= 64) return go(short_rows_kernel<E, 8, 8, true>, 8);
            if (p.V <= 256) return go(short_rows_kernel<E, 16, 16, true>, 16);
        }
        if (p.V <= 16) return go(short_rows_kernel<E, 4, 4, false>, 4);
        if (p.V <= 64) return go(short_rows_kernel<E, 8, 8, false>, 8);
        if (p.V <= 256) return go(short_rows_kernel<E, 16, 16, false>, 16);
        if (p.V <= 512) return go(short_rows_kernel<E, kWave, 8, false>, kWave);
        return go(short_rows_kernel<E, kWave, 32, false>, kWave);
    }
    const Cut cut = part_cut(p.R, p.V);
    p.parts = cut.parts;
    p.per = cut.per;
    if (!fits_a_launch((int64_t)p.R * p.parts, kThreads)) return MARL_ERR_BAD_DIM;
    hipLaunchKernelGGL(long_rows_kernel<E>, dim3((unsigned)(p.R * p.parts)), dim3(kThreads), 0, stream, p);
    if (p.parts > 1) hipLaunchKernelGGL(join_kernel<E>, dim3((unsigned)p.R), dim3(kWave), 0, stream, p);
    return launched("distill");
}

template <typename E>
int run_backward(DistillArgs p, hipStream_t stream)
{
    if (p.V <= kShort) {
        auto go = [&](auto kernel, int G) {
            const int64_t rows = (int64_t)(kThreads / kWave) * (kWave / G);
            hipLaunchKernelGGL(kernel, dim3((unsigned)((p.R + rows - 1) / rows)), dim3(kThreads), 0, stream, p);
            return launched("distill gradient");
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
    if (!fits_a_launch((int64_t)p.R * p.parts, kThreads)) return MARL_ERR_BAD_DIM;
    hipLaunchKernelGGL(long_grad_kernel<E>, dim3((unsigned)(p.R * p.parts)), dim3(kThreads), 0, stream, p);
    return launched("distill gradient");
}

}  // namespace
}  // namespace marl

using namespace marl;

extern "C" {

int marl_distill_workspace_bytes(int32_t R, int32_t V, int32_t K, size_t *bytes)
{
    if (!bytes) return MARL_ERR_NULL;
    if (R < 0 || V < 1 || V >= (1 << 30) || K < 1 || K > kMostKept || !rows_fit(R, V)) return MARL_ERR_BAD_DIM;
    *bytes = distill_workspace(R, V);
    return MARL_OK;
}

int marl_distill(int32_t dtype, int32_t R, int32_t V, int32_t K, const void *logits, int64_t ld, const int32_t *top_id,
                 const float *top_value, const uint8_t *avail, int64_t ld_avail, float scale, int32_t tail, float *loss,
                 float *log_sum, float *log_rest, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const int rc = logit_rows_check(dtype, R, V, logits, ld, avail, ld_avail, scale);
    if (rc) return rc;
    if (K < 1 || K > kMostKept || !rows_fit(R, V) || workspace_bytes < distill_workspace(R, V)) return MARL_ERR_BAD_DIM;
    if (R == 0) return MARL_OK;
    if (!top_id || !top_value || !loss || (workspace_bytes && !workspace)) return MARL_ERR_NULL;
    if (!aligned_to(workspace, 256)) return MARL_ERR_BAD_ARG;
    DistillArgs p{};
    p.R = R; p.V = V; p.K = K; p.tail = tail != 0;
    p.logits = logits; p.ld = ld; p.avail = avail; p.ld_avail = ld_avail; p.scale = scale; p.lowest = lowest_of(scale);
    p.top_id = top_id; p.top_value = top_value; p.loss = loss; p.log_sum = log_sum; p.log_rest = log_rest;
    p.stats = static_cast<float *>(workspace);
    return with_dtype(dtype, [&](auto e) { return run_forward<decltype(e)>(p, static_cast<hipStream_t>(hip_stream)); });
}

int marl_distill_grad(int32_t dtype, int32_t R, int32_t V, int32_t K, const void *logits, int64_t ld, const int32_t *top_id,
                      const float *top_value, const uint8_t *avail, int64_t ld_avail, float scale, int32_t tail, const float *log_sum,
                      const float *log_rest, const float *grad_loss, void *grad_logits, int64_t ld_grad, void *hip_stream)
{
    const int rc = logit_rows_check(dtype, R, V, logits, ld, avail, ld_avail, scale);
    if (rc) return rc;
    if (K < 1 || K > kMostKept || !rows_fit(R, V) || ld_grad < V) return MARL_ERR_BAD_DIM;
    if (grad_logits && grad_logits == logits && ld_grad != ld) return MARL_ERR_BAD_ARG;
    if (R == 0) return MARL_OK;
    if (!top_id || !top_value || !log_sum || (tail && !log_rest) || !grad_loss || !grad_logits) return MARL_ERR_NULL;
    DistillArgs p{};
    p.R = R; p.V = V; p.K = K; p.tail = tail != 0;
    p.logits = logits; p.ld = ld; p.avail = avail; p.ld_avail = ld_avail; p.scale = scale; p.lowest = lowest_of(scale);
    p.top_id = top_id; p.top_value = top_value; p.in_log_sum = log_sum; p.in_log_rest = log_rest; p.grad_loss = grad_loss;
    p.grad_logits = grad_logits; p.ld_grad = ld_grad;
    return with_dtype(dtype, [&](auto e) { return run_backward<decltype(e)>(p, static_cast<hipStream_t>(hip_stream)); });
}

}  // extern "C"
