// Rows over a vocabulary: log probabilities of tokens with entropy and alternatives, and distillation from top lists.
#pragma once
#include "op_common.h"
#include "../../../include/comp_ams_operators.h"

namespace cams_ops {

constexpr int kVocabThreads = 256;
constexpr int kMaxTop = COMP_AMS_MAX_TOP;

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

// --- the teacher's list of one row --------------------------------------------------------------------------------

struct Listed {
    int32_t token;       // -1: not there
    float q, logq;       // the token's share; its logarithm, 0 where the share is 0
    bool any;            // the row lists something
};

// Entry threadIdx.x of the row's list for the first kMaxTop threads (the others: not there).  Every thread of the workgroup
// calls this.  lds: kMaxTop floats.
__device__ __forceinline__ Listed teacher_entry(const int32_t *__restrict__ idx, const float *__restrict__ val, int64_t row, int k,
                                                int64_t vocab, float inv_t, float *lds)
{
    const int t = threadIdx.x;
    Listed e = {-1, 0.f, 0.f, false};
    float v = -INFINITY;
    if (t < k) {
        const int32_t tok = idx[row * k + t];
        if (tok >= 0 && tok < vocab) {
            e.token = tok;
            v = val[row * k + t] * inv_t;
        }
    }
    __syncthreads();
    if (t < kMaxTop) lds[t] = v;
    // a NaN marks "there": a list of entries of -infinity alone has no distribution either
    const int there = __syncthreads_or(e.token >= 0);
    e.any = there != 0;
    float top = -INFINITY;
    for (int q = 0; q < k; ++q) top = MaxOp::apply(top, lds[q]);
    float sum = 0.f;
    for (int q = 0; q < k; ++q) sum += __builtin_amdgcn_exp2f((lds[q] - top) * kLog2e);
    if (e.token >= 0) {
        e.q = __builtin_amdgcn_exp2f((v - top) * kLog2e) / sum;
        e.logq = e.q == 0.f ? 0.f : (v - top) - logf(sum);
    }
    return e;
}

struct DistillArgs {
    int64_t rows, vocab, in_stride, out_stride;
    int32_t k;
    float t, inv_t;          // the temperature and its reciprocal
};

// The row's loss from its list: every entry's share of T^2 sum q (log q - lp).  Every thread of the workgroup calls this.
template <typename T, int kThreads>
__device__ __forceinline__ float distill_loss(const Listed &e, const T *__restrict__ z, float lse, const DistillArgs &a, float *scratch)
{
    float part = 0.f;
    if (e.token >= 0 && e.q != 0.f) part = e.q * (e.logq - (widen1(z[e.token]) * a.inv_t - lse));
    return a.t * a.t * team_reduce<SumOp, kThreads>(part, scratch);
}

// What the listed tokens' gradients are corrected by: a token's share is the sum over the entries that name it, and the first
// of them writes.  Returns whether this thread does.  lds: kMaxTop tokens and shares.
__device__ __forceinline__ bool merged_share(const Listed &e, int k, int32_t *lds_token, float *lds_q, float *share)
{
    const int t = threadIdx.x;
    __syncthreads();
    if (t < kMaxTop) {
        lds_token[t] = t < k ? e.token : -1;
        lds_q[t] = e.q;
    }
    __syncthreads();
    if (e.token < 0) return false;
    bool first = true;
    float s = 0.f;
    for (int q = 0; q < k; ++q)
        if (lds_token[q] == e.token) {
            first = first && q >= t;
            s += lds_q[q];
        }
    *share = s;
    return first;
}

// Rows of any length: one workgroup per row.  kLoss: maximum and sum are formed (else lse is given); kGrad: the gradient is written.
template <typename T, bool kLoss, bool kGrad>
__global__ __launch_bounds__(kVocabThreads) void distill_any(float *__restrict__ loss, float *__restrict__ lse_out, T *dlogits,
                                                             const float *__restrict__ dloss, const T *logits,
                                                             const float *__restrict__ lse_in, const int32_t *__restrict__ idx,
                                                             const float *__restrict__ val, DistillArgs a)
{
    __shared__ Lse lse_scratch[kVocabThreads / kWave];
    __shared__ float scratch[kVocabThreads / kWave];
    __shared__ float list[kMaxTop];
    __shared__ int32_t list_token[kMaxTop];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *z = logits + row * a.in_stride;
        float lse;
        if constexpr (kLoss) {
            const float unit = a.inv_t * kLog2e;
            Lse v = {-INFINITY, 0.f};
            for (int64_t c = threadIdx.x; c < a.vocab; c += kVocabThreads) v = lse_join(v, {widen1(z[c]), 1.f}, unit);
            v = block_lse<kVocabThreads>(v, unit, lse_scratch);
            lse = lse_value(v, a.inv_t);
        } else {
            lse = lse_in[row];
        }
        const Listed e = teacher_entry(idx, val, row, a.k, a.vocab, a.inv_t, list);
        if constexpr (kLoss) {
            const float l = distill_loss<T, kVocabThreads>(e, z, lse, a, scratch);
            if (threadIdx.x == 0) {
                if (loss) loss[row] = e.any ? l : 0.f;
                if (lse_out) lse_out[row] = lse;
            }
        }
        if constexpr (kGrad) {
            T *out = dlogits + row * a.out_stride;
            const float w = e.any ? dloss[row] * a.t : 0.f;
            float share = 0.f, at_token = 0.f;
            const bool writes = merged_share(e, a.k, list_token, list, &share);
            if (writes) at_token = widen1(z[e.token]);         // before an in-place gradient replaces it
            __syncthreads();
            for (int64_t c = threadIdx.x; c < a.vocab; c += kVocabThreads)
                out[c] = narrow1<T>(e.any ? w * __builtin_amdgcn_exp2f(fmaf(widen1(z[c]), a.inv_t, -lse) * kLog2e) : 0.f);
            __syncthreads();
            if (writes) out[e.token] = narrow1<T>(w * (__builtin_amdgcn_exp2f(fmaf(at_token, a.inv_t, -lse) * kLog2e) - share));
        }
    }
}

}  // namespace cams_ops
