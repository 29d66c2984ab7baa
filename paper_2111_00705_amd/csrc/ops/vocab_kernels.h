// Rows over a vocabulary: log probabilities of tokens with entropy and alternatives, and distillation from top lists.
#pragma once
#include "op_common.h"
#include "../../../include/comp_ams_operators.h"

namespace cams_ops {

constexpr int kVocabThreads = 256;
constexpr int kMaxTop = COMP_AMS_MAX_TOP;

template <typename T> constexpr uint32_t kNegInfBits = sizeof(T) == 4 ? 0xff800000u : __is_same(T, bf16_t) ? 0xff80u : 0xfc00u;

// A logit's place in the order of the top list as one whole number: the larger value first, -0 as +0, every NaN above
// +infinity and equal to the others; among equals the lower token.
__device__ __forceinline__ uint32_t order_of(float z)
{
    if (z != z) return 0xffffffffu;
    const uint32_t b = __float_as_uint(z + 0.f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t rank_key(float z, uint32_t token) { return ((uint64_t)order_of(z) << 32) | (uint32_t)~token; }

template <int kThreads>
__device__ __forceinline__ Lse block_lse(Lse v, float unit, Lse *scratch)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = lse_join(v, {__shfl_xor(v.top, off, kWave), __shfl_xor(v.sum, off, kWave)}, unit);
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) scratch[threadIdx.x / kWave] = v;
    __syncthreads();
    v = scratch[0];
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) v = lse_join(v, scratch[w], unit);
    return v;
}

template <int kThreads>
__device__ __forceinline__ uint64_t block_max(uint64_t v, uint64_t *scratch)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = max(v, (uint64_t)__shfl_xor((unsigned long long)v, off, kWave));
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) scratch[threadIdx.x / kWave] = v;
    __syncthreads();
    v = scratch[0];
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) v = max(v, scratch[w]);
    return v;
}

// Rows of any length: the row is read for maximum and sum, for the entropy, and once more for each alternative.
template <typename T>
__global__ __launch_bounds__(kVocabThreads) void logprobs_any(float *__restrict__ logp, float *__restrict__ entropy,
                                                              int32_t *__restrict__ top_idx, float *__restrict__ top_logp,
                                                              const T *__restrict__ logits, const int64_t *__restrict__ tokens,
                                                              int64_t rows, int64_t vocab, int64_t stride, int k)
{
    __shared__ Lse lse_scratch[kVocabThreads / kWave];
    __shared__ float scratch[kVocabThreads / kWave];
    __shared__ uint64_t key_scratch[kVocabThreads / kWave];
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T *z = logits + row * stride;
        Lse v = {-INFINITY, 0.f};
        for (int64_t c = threadIdx.x; c < vocab; c += kVocabThreads) v = lse_join(v, {widen1(z[c]), 1.f}, kLog2e);
        v = block_lse<kVocabThreads>(v, kLog2e, lse_scratch);
        const float lse = lse_value(v, 1.f);
        float e = 0.f;
        for (int64_t c = threadIdx.x; c < vocab; c += kVocabThreads) {
            const float zc = widen1(z[c]), p = __builtin_amdgcn_exp2f((zc - lse) * kLog2e);
            if (p != 0.f) e = fmaf(p, lse - zc, e);
        }
        e = team_reduce<SumOp, kVocabThreads>(e, scratch);
        if (threadIdx.x == 0) {
            if (entropy) entropy[row] = e;
            if (logp) {
                const int64_t t = tokens[row];
                logp[row] = t >= 0 && t < vocab ? widen1(z[t]) - lse : 0.f;
            }
        }
        uint64_t last = ~0ull;
        for (int q = 0; q < k; ++q) {
            uint64_t best = 0;
            for (int64_t c = threadIdx.x; c < vocab; c += kVocabThreads) {
                const uint64_t key = rank_key(widen1(z[c]), (uint32_t)c);
                if (key < last) best = max(best, key);
            }
            last = block_max<kVocabThreads>(best, key_scratch);
            if (threadIdx.x == 0) {
                const uint32_t t = ~(uint32_t)last;
                top_idx[row * k + q] = (int32_t)t;
                top_logp[row * k + q] = widen1(z[t]) - lse;
            }
        }
    }
}

// The logit of a rank key (-0 comes back as +0).
__device__ __forceinline__ float logit_of(uint64_t key)
{
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}

// Statistics of a piece of a row: top = max z, sum = sum exp(z - top), moment = sum exp(z - top) (z - top).  The entropy of the
// distribution is log sum - moment / sum: no cancellation against lse.
struct Piece {
    float top, sum, moment;
};
__device__ __forceinline__ Piece piece_join(const Piece &a, const Piece &b)
{
    const float top = MaxOp::apply(a.top, b.top);
    const float da = a.top - top, db = b.top - top;
    const float fa = a.top == top ? 1.f : __builtin_amdgcn_exp2f(da * kLog2e);
    const float fb = b.top == top ? 1.f : __builtin_amdgcn_exp2f(db * kLog2e);
    // an empty piece (top -infinity, sum 0) adds nothing, though its distance is infinite
    const float ma = a.top == top ? a.moment : fa == 0.f ? 0.f : fa * fmaf(da, a.sum, a.moment);
    const float mb = b.top == top ? b.moment : fb == 0.f ? 0.f : fb * fmaf(db, b.sum, b.moment);
    return {top, a.sum * fa + b.sum * fb, ma + mb};
}

constexpr int kMaxCandidates = 1024;      // of one piece; more than that (rows of ties) are told apart by select_slow
constexpr int kMaxPieces = 32;            // of one row; longer vocabularies go to logprobs_any

// Adds the k tokens of the largest keys of z[lo..hi) to the list by bisection over the order and, among the ties at its end,
// over the token; the piece is read once for each bit.  Every thread of the workgroup calls this; hi - lo >= k >= 1.
template <typename T, int kThreads>
__device__ __attribute__((noinline)) void select_slow(const T *z, int64_t lo, int64_t hi, int k, uint64_t *list, uint32_t *count)
{
    __shared__ uint32_t counts[2];
    uint32_t at = 0;
    int turn = 0;
    auto counted = [&](auto &&test) {
        uint32_t mine = 0;
        for (int64_t c = lo + threadIdx.x; c < hi; c += kThreads) mine += test(order_of(widen1(z[c])), (uint32_t)c) ? 1u : 0u;
        if (threadIdx.x == 0) counts[turn] = 0;
        __syncthreads();
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) mine += __shfl_xor(mine, off, kWave);
        if ((threadIdx.x & (kWave - 1)) == 0) atomicAdd(&counts[turn], mine);       // whole numbers: the order does not matter
        __syncthreads();
        const uint32_t all = counts[turn];
        turn ^= 1;
        return all;
    };
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t more = at | (1u << bit);
        if (counted([&](uint32_t o, uint32_t) { return o >= more; }) >= (uint32_t)k) at = more;
    }
    const uint32_t above = counted([&](uint32_t o, uint32_t) { return o > at; });
    const uint32_t ties = (uint32_t)k - above;             // at least one: `at` is the k-th largest
    uint32_t last = 0;                                       // the largest token of which fewer than `ties` ties come before it
    for (int bit = 30; bit >= 0; --bit) {
        const uint32_t more = last | (1u << bit);
        if (counted([&](uint32_t o, uint32_t c) { return o == at && c < more; }) < ties) last = more;
    }
    if (threadIdx.x == 0) *count = 0;
    __syncthreads();
    for (int64_t c = lo + threadIdx.x; c < hi; c += kThreads) {
        const uint32_t o = order_of(widen1(z[c]));
        if (o > at || (o == at && (uint32_t)c <= last)) list[atomicAdd(count, 1u)] = ((uint64_t)o << 32) | (uint32_t)~(uint32_t)c;
    }
    __syncthreads();
}

// One piece of a row per workgroup, held in registers between the two looks at it: maximum, sum and moment, and then the
// elements that can be among the k best.  Those are found by a bound: the k-th largest of the maxima of `groups` groups of lanes is
// reached by k elements at least, and by few more (k = 32 of 64 groups: 44 expected), which are listed in LDS and ranked by counting.
// With one piece per row the results are final; with more, statistics and keys go to work and logprobs_join follows.
template <typename T, int kThreads, int kVecs>
__global__ __launch_bounds__(kThreads) void logprobs_regs(float *__restrict__ logp, float *__restrict__ entropy,
                                                          int32_t *__restrict__ top_idx, float *__restrict__ top_logp,
                                                          const T *__restrict__ logits, const int64_t *__restrict__ tokens,
                                                          int64_t vocab, int64_t stride, int k, int groups, int n_pieces,
                                                          int64_t piece_len, Piece *__restrict__ pieces, uint64_t *__restrict__ keys)
{
    constexpr int E = kVec<T>;
    __shared__ float scratch[kThreads / kWave], scratch2[kThreads / kWave];
    __shared__ float group_max[256];
    __shared__ uint64_t list[kMaxCandidates];
    __shared__ uint32_t count;
    __shared__ float bound_lds;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x / (unsigned)n_pieces, lo = blockIdx.x % (unsigned)n_pieces * piece_len;
    const int len = (int)(min(lo + piece_len, vocab) - lo);
    const T *z = logits + row * stride + lo;
    v4u raw[kVecs];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) raw[v] = load_row(z, (v * kThreads + tid) * E, len, kNegInfBits<T>);
    float vec_max[kVecs], top = -INFINITY;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        float x[E];
        widen<T>(raw[v], x);
        vec_max[v] = x[0];
#pragma unroll
        for (int q = 1; q < E; ++q) vec_max[v] = fmaxf(vec_max[v], x[q]);      // ignores NaN: the sum shows them
        top = fmaxf(top, vec_max[v]);
    }
    // group maxima on the way to the workgroup's
    if (k > 0) {
        const int per = kThreads / groups;
        float g = top;
        for (int off = 1; off < per; off <<= 1) g = fmaxf(g, __shfl_xor(g, off, kWave));
        if ((tid & (per - 1)) == 0) group_max[tid / per] = g;
        if (tid == 0) count = 0;
    }
    const float m = team_reduce<MaxOp, kThreads>(top, scratch);
    float s = 0.f, w = 0.f;
    if (m != -INFINITY) {
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            float x[E];
            rewiden(raw[v]);
            widen<T>(raw[v], x);
#pragma unroll
            for (int q = 0; q < E; ++q) {
                const float d = x[q] - m, e = __builtin_amdgcn_exp2f(d * kLog2e);
                s += e;
                w = fmaf(e, fmaxf(d, -1e30f), w);       // an infinite distance has e = 0
            }
        }
    } else {
#pragma unroll 1
        for (int c = tid; c < len; c += kThreads) {     // nothing but -infinity, or NaN, which must show
            const float x = widen1(z[c]);
            if (x != x) s = x;
        }
    }
    float bound = -INFINITY;
    if (k > 0) {
        if (tid < groups) {
            const float g = group_max[tid];
            int rank = 0;
            for (int q = 0; q < groups; ++q) {
                const float o = group_max[q];
                rank += (o > g || (o == g && q < tid)) ? 1 : 0;
            }
            if (rank == k - 1) bound_lds = g;
        }
    }
    const float sum = team_reduce<SumOp, kThreads>(s, scratch2);
    const float moment = team_reduce<SumOp, kThreads>(w, scratch);
    if (k > 0) {
        bound = bound_lds;
        if (sum == sum) {
#pragma unroll
            for (int v = 0; v < kVecs; ++v) {
                if (vec_max[v] >= bound) {
                    float x[E];
                    rewiden(raw[v]);
                    widen<T>(raw[v], x);
#pragma unroll
                    for (int q = 0; q < E; ++q) {
                        const int c = (v * kThreads + tid) * E + q;
                        if (x[q] >= bound && c < len) {
                            const uint32_t slot = atomicAdd(&count, 1u);
                            if (slot < (uint32_t)kMaxCandidates) list[slot] = rank_key(x[q], (uint32_t)(lo + c));
                        }
                    }
                }
            }
        }
        __syncthreads();
        // a NaN or +infinity (the bound says nothing then), or too many ties
        if (sum != sum || count > (uint32_t)kMaxCandidates) {
            __syncthreads();
            if (len > k) {
                select_slow<T, kThreads>(logits + row * stride, lo, lo + len, k, list, &count);
            } else {
                if (tid == 0) count = (uint32_t)len;
                for (int c = tid; c < len; c += kThreads) list[c] = rank_key(widen1(z[c]), (uint32_t)(lo + c));
                __syncthreads();
            }
        }
    }
    const bool whole = n_pieces == 1;
    const float lse = fabsf(m) == INFINITY ? NAN : m + logf(sum);
    if (tid == 0) {
        if (!whole) {
            pieces[blockIdx.x] = {m, sum, moment};
        } else {
            if (entropy) entropy[row] = fabsf(m) == INFINITY ? NAN : logf(sum) - moment / sum;
            if (logp) {
                const int64_t t = tokens[row];
                logp[row] = t >= 0 && t < vocab ? widen1(logits[row * stride + t]) - lse : 0.f;
            }
        }
    }
    const int n = k > 0 ? (int)count : 0;
    for (int t = tid; t < n; t += kThreads) {
        const uint64_t key = list[t];
        int rank = 0;
        for (int q = 0; q < n; ++q) rank += list[q] > key ? 1 : 0;
        if (rank < k) {
            if (whole) {
                top_idx[row * k + rank] = (int32_t)~(uint32_t)key;
                top_logp[row * k + rank] = logit_of(key) - lse;
            } else {
                keys[(int64_t)blockIdx.x * k + rank] = key;
            }
        }
    }
    if (!whole)
        for (int t = n + tid; t < k; t += kThreads) keys[(int64_t)blockIdx.x * k + t] = 0;   // a short last piece
}

// The pieces of a row: statistics joined in order, their best tokens ranked against each other.
template <typename T>
__global__ __launch_bounds__(kVocabThreads) void logprobs_join(float *__restrict__ logp, float *__restrict__ entropy,
                                                               int32_t *__restrict__ top_idx, float *__restrict__ top_logp,
                                                               const T *__restrict__ logits, const int64_t *__restrict__ tokens,
                                                               int64_t vocab, int64_t stride, int k, int n_pieces,
                                                               const Piece *__restrict__ pieces, const uint64_t *__restrict__ keys)
{
    extern __shared__ uint64_t list[];
    const int64_t row = blockIdx.x;
    const int n = n_pieces * k;
    for (int t = threadIdx.x; t < n; t += kVocabThreads) list[t] = keys[row * n + t];
    Piece p = pieces[row * n_pieces];
    for (int q = 1; q < n_pieces; ++q) p = piece_join(p, pieces[row * n_pieces + q]);
    const bool none = fabsf(p.top) == INFINITY;
    const float lse = none ? NAN : p.top + logf(p.sum);
    if (threadIdx.x == 0) {
        if (entropy) entropy[row] = none ? NAN : logf(p.sum) - p.moment / p.sum;
        if (logp) {
            const int64_t t = tokens[row];
            logp[row] = t >= 0 && t < vocab ? widen1(logits[row * stride + t]) - lse : 0.f;
        }
    }
    __syncthreads();
    for (int t = threadIdx.x; t < n; t += kVocabThreads) {
        const uint64_t key = list[t];
        int rank = 0;
        for (int q = 0; q < n; ++q) rank += list[q] > key ? 1 : 0;
        if (rank < k && key) {
            top_idx[row * k + rank] = (int32_t)~(uint32_t)key;
            top_logp[row * k + rank] = logit_of(key) - lse;
        }
    }
}

// --- distillation -------------------------------------------------------------------------------------------------

struct DistillArgs {
    int64_t rows, vocab, in_stride, out_stride;
    int32_t k;
    float t, inv_t;          // the temperature and its reciprocal
};

// The teacher's list of one row, two entries in each lane of a wavefront: every wavefront that needs the list forms its shares for
// itself, without a barrier.
struct Listed {
    int32_t token[2];    // -1: not there
    float q[2];          // the tokens' shares
    float logq[2];       // their logarithms, 0 where the share is 0
    bool any;            // the row lists something
};
static_assert(kMaxTop <= 2 * kWave, "two entries per lane");

__device__ __forceinline__ Listed teacher_list(const int32_t *__restrict__ idx, const float *__restrict__ val, int64_t row,
                                               const DistillArgs &a)
{
    const int lane = threadIdx.x & (kWave - 1);
    Listed e;
    float v[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int t = lane + u * kWave;
        e.token[u] = -1;
        v[u] = -INFINITY;
        if (t < a.k) {
            const int32_t tok = idx[row * a.k + t];
            const float x = val[row * a.k + t] * a.inv_t;
            if (tok >= 0 && tok < a.vocab) {
                e.token[u] = tok;
                v[u] = x;
            }
        }
    }
    e.any = __ballot(e.token[0] >= 0 || e.token[1] >= 0) != 0;
    const float top = lanes_reduce<MaxOp, kWave>(MaxOp::apply(v[0], v[1]));
    float x[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) x[u] = e.token[u] >= 0 ? __builtin_amdgcn_exp2f((v[u] - top) * kLog2e) : 0.f;
    const float sum = lanes_reduce<SumOp, kWave>(x[0] + x[1]), log_sum = logf(sum);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        e.q[u] = x[u] == 0.f ? 0.f : x[u] / sum;
        e.logq[u] = e.q[u] == 0.f ? 0.f : (v[u] - top) - log_sum;
    }
    return e;
}

// T^2 sum q (log q - lp) of the row, by one wavefront.
template <typename T>
__device__ __forceinline__ float list_loss(const Listed &e, const T *z, float lse, const DistillArgs &a)
{
    float part = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u)
        if (e.q[u] != 0.f) part += e.q[u] * (e.logq[u] - fmaf(widen1(z[e.token[u]]), a.inv_t, -lse));
    return a.t * a.t * lanes_reduce<SumOp, kWave>(part);
}

// What stands at the listed tokens, by one wavefront: q[u] becomes the sum over the entries that name the token, and token[u] is -1
// but for the first of them.
__device__ __forceinline__ void merge_list(Listed &e, int k)
{
    const int lane = threadIdx.x & (kWave - 1);
    float share[2] = {0.f, 0.f};
    bool first[2] = {true, true};
    for (int t = 0; t < k; ++t) {
        const int u = t >> 6;
        const int32_t token = __builtin_amdgcn_readlane(u ? e.token[1] : e.token[0], t & (kWave - 1));
        const float q = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(u ? e.q[1] : e.q[0]), t & (kWave - 1)));
#pragma unroll
        for (int w = 0; w < 2; ++w)
            if (token == e.token[w]) {
                share[w] += q;
                first[w] = first[w] && t >= lane + w * kWave;
            }
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        e.q[w] = share[w];
        if (!first[w]) e.token[w] = -1;
    }
}

// Maximum and sum of a row's elements [at, at + kVecs kThreads E) taken into this thread's (top, sum).
template <typename T, int kThreads, int kVecs>
__device__ __forceinline__ void take_chunk(Lse &v, v4u (&raw)[kVecs], float unit)
{
    constexpr int E = kVec<T>;
    float top = v.top;
#pragma unroll
    for (int r = 0; r < kVecs; ++r) {
        float x[E];
        widen<T>(raw[r], x);
#pragma unroll
        for (int q = 0; q < E; ++q) top = fmaxf(top, x[q]);     // ignores NaN: the sum shows them
    }
    const float from = top == -INFINITY ? 0.f : top;            // nothing but -infinity so far: exponentials of zero, not of NaN
    float s = v.sum * __builtin_amdgcn_exp2f((v.top - from) * unit);
#pragma unroll
    for (int r = 0; r < kVecs; ++r) {
        float x[E];
        rewiden(raw[r]);
        widen<T>(raw[r], x);
#pragma unroll
        for (int q = 0; q < E; ++q) s += __builtin_amdgcn_exp2f((x[q] - from) * unit);
    }
    v = {top, s};
}

// The loss: one pass over the row with a running maximum and sum, four vectors a thread in flight.
template <typename T, int kThreads>
__global__ __launch_bounds__(kThreads) void distill_forward(float *__restrict__ loss, float *__restrict__ lse_out,
                                                            const T *__restrict__ logits, const int32_t *__restrict__ idx,
                                                            const float *__restrict__ val, DistillArgs a)
{
    constexpr int E = kVec<T>, kVecs = 4;
    __shared__ Lse lse_scratch[kThreads / kWave];
    const int64_t row = blockIdx.x;
    const T *z = logits + row * a.in_stride;
    Lse v = {-INFINITY, 0.f};
    for (int64_t at = 0; at < a.vocab; at += (int64_t)kVecs * kThreads * E) {
        v4u raw[kVecs];
#pragma unroll
        for (int r = 0; r < kVecs; ++r) raw[r] = load_row(z, at + (r * kThreads + (int)threadIdx.x) * E, a.vocab, kNegInfBits<T>);
        take_chunk<T, kThreads, kVecs>(v, raw, a.inv_t * kLog2e);
    }
    const float lse = lse_value(block_lse<kThreads>(v, a.inv_t * kLog2e, lse_scratch), a.inv_t);
    if (threadIdx.x < kWave) {
        const Listed e = teacher_list(idx, val, row, a);
        const float l = list_loss(e, z, lse, a);
        if (threadIdx.x == 0) {
            if (loss) loss[row] = e.any ? l : 0.f;
            if (lse_out) lse_out[row] = lse;
        }
    }
}

// The gradient from a given lse: a piece of a row per workgroup.
template <typename T, int kThreads>
__global__ __launch_bounds__(kThreads) void distill_gradient(T *dlogits, const float *__restrict__ dloss, const T *logits,
                                                             const float *__restrict__ lse_in, const int32_t *__restrict__ idx,
                                                             const float *__restrict__ val, DistillArgs a, int n_pieces, int64_t piece_len)
{
    constexpr int E = kVec<T>, kVecs = 4;
    const int64_t row = blockIdx.x / (unsigned)n_pieces, lo = blockIdx.x % (unsigned)n_pieces * piece_len;
    const int64_t hi = min(lo + piece_len, a.vocab);
    const T *z = logits + row * a.in_stride;
    T *out = dlogits + row * a.out_stride;
    const float lse = lse_in[row];
    Listed e = teacher_list(idx, val, row, a);
    const float w = dloss[row] * a.t;
    auto gradient = [&](float x) { return e.any ? w * __builtin_amdgcn_exp2f(fmaf(x, a.inv_t, -lse) * kLog2e) : 0.f; };
    float listed[2] = {0.f, 0.f};
    if (threadIdx.x < kWave) {
        merge_list(e, a.k);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (e.token[u] < lo || e.token[u] >= hi) e.token[u] = -1;
            if (e.token[u] >= 0) listed[u] = widen1(z[e.token[u]]);        // before an in-place gradient replaces it
        }
    }
    __syncthreads();
    for (int64_t at = lo; at < hi; at += (int64_t)kVecs * kThreads * E) {
        v4u raw[kVecs];
#pragma unroll
        for (int r = 0; r < kVecs; ++r) raw[r] = load_row(z, at + (r * kThreads + (int)threadIdx.x) * E, hi);
#pragma unroll
        for (int r = 0; r < kVecs; ++r) {
            float x[E];
            widen<T>(raw[r], x);
#pragma unroll
            for (int q = 0; q < E; ++q) x[q] = gradient(x[q]);
            store_row(out, at + (r * kThreads + (int)threadIdx.x) * E, hi, narrow<T>(x));
        }
    }
    __syncthreads();
    if (threadIdx.x < kWave) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (e.token[u] >= 0) {
                const float p = __builtin_amdgcn_exp2f(fmaf(listed[u], a.inv_t, -lse) * kLog2e);
                out[e.token[u]] = narrow1<T>(w * (p - e.q[u]));
            }
    }
}

// Loss and gradient at once.  kVecs > 0: the row stays in registers, kVecs vectors a thread, and is read once.  kVecs = 0: rows of
// any length, read a second time for the gradient.
template <typename T, int kThreads, int kVecs>
__global__ __launch_bounds__(kThreads) void distill_both(float *__restrict__ loss, T *dlogits, const float *__restrict__ dloss,
                                                         const T *logits, const int32_t *__restrict__ idx, const float *__restrict__ val,
                                                         DistillArgs a)
{
    constexpr int E = kVec<T>, kHeld = kVecs ? kVecs : 4;
    constexpr int64_t kChunk = (int64_t)kHeld * kThreads * E;
    __shared__ Lse lse_scratch[kThreads / kWave];
    const int64_t row = blockIdx.x;
    const T *z = logits + row * a.in_stride;
    T *out = dlogits + row * a.out_stride;
    const float unit = a.inv_t * kLog2e;
    auto place = [&](int64_t at, int r) { return at + (r * kThreads + (int)threadIdx.x) * E; };
    Lse v = {-INFINITY, 0.f};
    v4u raw[kHeld];
    for (int64_t at = 0; at < (kVecs ? 1 : a.vocab); at += kChunk) {
#pragma unroll
        for (int r = 0; r < kHeld; ++r) raw[r] = load_row(z, place(at, r), a.vocab, kNegInfBits<T>);
        take_chunk<T, kThreads, kHeld>(v, raw, unit);
    }
    v = block_lse<kThreads>(v, unit, lse_scratch);
    Listed e = teacher_list(idx, val, row, a);
    const float w = dloss[row] * a.t, scale = w / v.sum;
    auto gradient = [&](float x) { return e.any ? scale * __builtin_amdgcn_exp2f((x - v.top) * unit) : 0.f; };
    float listed[2] = {0.f, 0.f};
    if (threadIdx.x < kWave) {
        const float l = list_loss(e, z, lse_value(v, a.inv_t), a);
        if (threadIdx.x == 0 && loss) loss[row] = e.any ? l : 0.f;
        merge_list(e, a.k);
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (e.token[u] >= 0) listed[u] = widen1(z[e.token[u]]);        // before an in-place gradient replaces it
    }
    __syncthreads();
    for (int64_t at = 0; at < (kVecs ? 1 : a.vocab); at += kChunk) {
        if constexpr (kVecs == 0) {
#pragma unroll
            for (int r = 0; r < kHeld; ++r) raw[r] = load_row(z, place(at, r), a.vocab);
        }
#pragma unroll
        for (int r = 0; r < kHeld; ++r) {
            float x[E];
            rewiden(raw[r]);
            widen<T>(raw[r], x);
#pragma unroll
            for (int q = 0; q < E; ++q) x[q] = gradient(x[q]);
            store_row(out, place(at, r), a.vocab, narrow<T>(x));
        }
    }
    __syncthreads();                                                       // the row is written before its listed tokens are
    if (threadIdx.x < kWave) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (e.token[u] >= 0)
                out[e.token[u]] = narrow1<T>(scale * __builtin_amdgcn_exp2f((listed[u] - v.top) * unit) - w * e.q[u]);
    }
}

}  // namespace cams_ops
