// Softmax of attention scores with a learned relative position bias, forward and backward.
#pragma once
#include "op_common.h"
#include "../../../include/comp_ams_operators.h"

namespace cams_ops {

// Bucket boundaries travel with the launch: strictly ascending, n_buckets - 1 of them.
struct Bounds {
    int32_t n;
    int32_t at[COMP_AMS_MAX_BUCKETS - 1];
};

struct BiasArgs {
    int64_t heads, tq, tk, rows;          // rows = batch heads tq
    int64_t s_b, s_h, s_q;                // strides of what is read first: the scores; dp
    int64_t p_b, p_h, p_q;                // the probabilities
    int64_t o_b, o_h, o_q;                // ds
    int64_t offset;
    float scale;
    int32_t causal;
};

constexpr int kBiasThreads = 256;

// How many of the bounds are <= r.
__device__ __forceinline__ int bucket_of(int64_t r, const int32_t *at, int n)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (at[mid] <= r) lo = mid + 1; else hi = mid;
    }
    return lo;
}

struct RowPlace {
    int64_t b, h, i;
};
__device__ __forceinline__ RowPlace place_of(int64_t row, const BiasArgs &a)
{
    const int64_t bh = row / a.tq;
    return {bh / a.heads, bh % a.heads, row % a.tq};
}

// Keys [0, seen) are those that query i of sequence b sees.
__device__ __forceinline__ int64_t keys_seen(const RowPlace &w, const int32_t *key_len, const BiasArgs &a)
{
    int64_t seen = a.tk;
    if (key_len) seen = min(seen, (int64_t)max(key_len[w.b], 0));
    if (a.causal) seen = min(seen, max(w.i + a.offset + 1, (int64_t)0));
    return seen;
}

// Rows of any length: one workgroup per row, which it reads three times (maximum, sum, result).
template <typename T>
__global__ __launch_bounds__(kBiasThreads) void bias_forward_any(T *p, const T *s, const float *__restrict__ table, Bounds bounds,
                                                                 const int32_t *__restrict__ key_len, BiasArgs a)
{
    __shared__ float scratch[kBiasThreads / kWave];
    __shared__ int32_t at[COMP_AMS_MAX_BUCKETS];
    __shared__ float bias[COMP_AMS_MAX_BUCKETS];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const RowPlace w = place_of(row, a);
        const int64_t seen = keys_seen(w, key_len, a);
        __syncthreads();
        for (int q = threadIdx.x; q <= bounds.n; q += kBiasThreads) {
            if (q < bounds.n) at[q] = bounds.at[q];
            bias[q] = table[q * a.heads + w.h];
        }
        __syncthreads();
        const T *sr = s + w.b * a.s_b + w.h * a.s_h + w.i * a.s_q;
        T *pr = p + w.b * a.p_b + w.h * a.p_h + w.i * a.p_q;
        auto score = [&](int64_t j) { return fmaf(widen1(sr[j]), a.scale, bias[bucket_of(j - w.i - a.offset, at, bounds.n)]); };
        float top = -INFINITY;
        for (int64_t j = threadIdx.x; j < seen; j += kBiasThreads) top = MaxOp::apply(top, score(j));
        top = team_reduce<MaxOp, kBiasThreads>(top, scratch);
        const bool none = top == -INFINITY;
        float sum = 0.f;
        if (!none)
            for (int64_t j = threadIdx.x; j < seen; j += kBiasThreads) sum += __builtin_amdgcn_exp2f((score(j) - top) * kLog2e);
        sum = team_reduce<SumOp, kBiasThreads>(sum, scratch);
        const float inv = 1.f / sum;
        for (int64_t j = threadIdx.x; j < a.tk; j += kBiasThreads)
            pr[j] = narrow1<T>(j < seen && !none ? __builtin_amdgcn_exp2f((score(j) - top) * kLog2e) * inv : 0.f);
    }
}

// Rows of any length, backward: a workgroup takes kBiasAnyRows queries of one head and sequence; first their sums of p dp, then
// the gradients, the bucket sums of each thread's keys going into the thread's own slots of LDS.
constexpr int kBiasAnyRows = 16;
constexpr int kBiasAnyThreads = 64;

template <typename T>
__global__ __launch_bounds__(kBiasAnyThreads) void bias_backward_any(T *ds, float *__restrict__ work, const T *dp, const T *__restrict__ p,
                                                                     Bounds bounds, const int32_t *__restrict__ key_len, BiasArgs a,
                                                                     int64_t pieces)
{
    __shared__ int32_t at[COMP_AMS_MAX_BUCKETS];
    __shared__ float slot[COMP_AMS_MAX_BUCKETS * kBiasAnyThreads];
    const int lane = threadIdx.x;
    const int64_t bh = blockIdx.x / pieces, piece = blockIdx.x % pieces;
    for (int q = lane; q < bounds.n; q += kBiasAnyThreads) at[q] = bounds.at[q];
    for (int q = 0; q <= bounds.n; ++q) slot[q * kBiasAnyThreads + lane] = 0.f;
    __syncthreads();
    for (int64_t i = piece * kBiasAnyRows; i < min((piece + 1) * kBiasAnyRows, a.tq); ++i) {
        const RowPlace w = {bh / a.heads, bh % a.heads, i};
        const int64_t seen = keys_seen(w, key_len, a);
        const T *pr = p + w.b * a.p_b + w.h * a.p_h + i * a.p_q, *dr = dp + w.b * a.s_b + w.h * a.s_h + i * a.s_q;
        T *or_ = ds + w.b * a.o_b + w.h * a.o_h + i * a.o_q;
        float sum = 0.f;
        for (int64_t j = lane; j < seen; j += kBiasAnyThreads) {
            const float pj = widen1(pr[j]);
            if (pj != 0.f) sum = fmaf(pj, widen1(dr[j]), sum);
        }
        sum = lanes_reduce<SumOp, kWave>(sum);
        for (int64_t j = lane; j < a.tk; j += kBiasAnyThreads) {
            float dt = 0.f;
            if (j < seen) {
                const float pj = widen1(pr[j]);
                if (pj != 0.f) dt = pj * (widen1(dr[j]) - sum);
                slot[bucket_of(j - i - a.offset, at, bounds.n) * kBiasAnyThreads + lane] += dt;
            }
            or_[j] = narrow1<T>(dt * a.scale);
        }
    }
    for (int q = 0; q <= bounds.n; ++q) {
        const float s = lanes_reduce<SumOp, kWave>(slot[q * kBiasAnyThreads + lane]);
        if (lane == 0) work[(int64_t)blockIdx.x * (bounds.n + 1) + q] = s;
    }
}

// work[batch][heads][pieces][buckets] -> dtable[worker][buckets][heads]; one wavefront per (bucket, head, worker), lanes in a
// fixed order.
template <typename G>
__global__ __launch_bounds__(kWave) void bias_table_join(G *__restrict__ dtable, const float *__restrict__ work, int64_t heads,
                                                         int64_t worker_batch, int64_t pieces, int buckets, int64_t grad_stride)
{
    const int64_t w = blockIdx.z, h = blockIdx.y, q = blockIdx.x;
    float s = 0.f;
    for (int64_t t = threadIdx.x; t < worker_batch * pieces; t += kWave) {
        const int64_t b = w * worker_batch + t / pieces, piece = t % pieces;
        s += work[((b * heads + h) * pieces + piece) * buckets + q];
    }
    s = lanes_reduce<SumOp, kWave>(s);
    if (threadIdx.x == 0) dtable[w * grad_stride + q * heads + h] = narrow1<G>(s);
}

}  // namespace cams_ops
