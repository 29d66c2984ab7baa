// Softmax of attention scores with a learned relative position bias, forward and backward.
//
//   t_ij = scale s_ij + table[bucket(j - i - offset)][head],  p = softmax_j(t) over the keys seen;
//   dt = p (dp - sum_j p dp),  ds = scale dt,  dtable[bucket] = sum of dt over the places in the bucket
//
// HBM-bound: scores are read once and probabilities written once; backward reads p and dp once, writes ds, and sums the table's gradient
// on the way.  Bias and gradient belong to relative positions, that is to diagonals: forward finds a row's biases side by side in LDS,
// backward adds up diagonals in registers.  Only the keys that a row sees are read.
// Measured (us of a pass among others, TB/s of what it cannot do without; a copy reaches 6.1): 16 x 12 x 512 x 512 bf16, lengths 0 to 512, forward
// 31.7 (4.6), backward 47.6 with the join (4.1); causal 2 x 16 x 1999 x 1999 f16 forward 113 (3.4), backward 113 (4.5).  Backward spends 25 of its
// 45 us in vector instructions (19 for each element, the reductions of a row among them); the rest is latency that two rows in flight a wavefront
// leave.
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
    bool stream_out;                      // p, ds are stored as a stream
    unsigned first;                       // workgroups that earlier launches of the call have taken
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
    __shared__ float scratch[kBiasThreads / kWave], scratch2[kBiasThreads / kWave];
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
        sum = team_reduce<SumOp, kBiasThreads>(sum, scratch2);
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
                                                                     int64_t pieces, int64_t worker_batch)
{
    __shared__ int32_t at[COMP_AMS_MAX_BUCKETS];
    __shared__ float slot[COMP_AMS_MAX_BUCKETS * kBiasAnyThreads];
    const int lane = threadIdx.x;
    const unsigned block = a.first + blockIdx.x;
    const int64_t bh = block / pieces, piece = block % pieces;
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
    const int64_t b = bh / a.heads, w = b / worker_batch, parts = worker_batch * pieces;
    for (int q = 0; q <= bounds.n; ++q) {
        const float s = lanes_reduce<SumOp, kWave>(slot[q * kBiasAnyThreads + lane]);
        if (lane == 0) work[((w * a.heads + bh % a.heads) * (bounds.n + 1) + q) * parts + (b - w * worker_batch) * pieces + piece] = s;
    }
}

// --- rows that a team of lanes holds in registers -----------------------------------------------------------------------

// What query i of the workgroup's (sequence, head) sees, as keys [0, seen).
__device__ __forceinline__ int row_seen(int64_t i, int64_t seen_by_length, const BiasArgs &a)
{
    int64_t seen = seen_by_length;
    if (a.causal) seen = min(seen, max(i + a.offset + 1, (int64_t)0));
    return (int)seen;
}

// Forward: a workgroup takes `rows_block` queries of one head and sequence, its teams in turn.  The head's bias over the relative
// positions that occur there is laid out in LDS first, [tk + rows_block - 1] floats in units of log 2, so that a vector of keys finds its
// biases side by side.
template <typename T, int kTeam, int kVecs>
__global__ __launch_bounds__(kTeamBlock<kTeam>) void bias_forward(T *p, const T *s, const float *__restrict__ table, Bounds bounds,
                                                                const int32_t *__restrict__ key_len, BiasArgs a, int pieces, int rows_block)
{
    constexpr int E = kVec<T>, kTeams = kTeamBlock<kTeam> / kTeam;
    extern __shared__ float along[];
    __shared__ float scratch[kTeamBlock<kTeam> / kWave], scratch2[kTeamBlock<kTeam> / kWave];
    __shared__ int32_t at[COMP_AMS_MAX_BUCKETS];
    __shared__ float of_bucket[COMP_AMS_MAX_BUCKETS];
    const Team<kTeam> me;
    // with a causal mask the last queries see most: they are taken first
    const unsigned block = a.first + blockIdx.x, bh = block / (unsigned)pieces, turn_of = block % (unsigned)pieces;
    const unsigned piece = a.causal ? pieces - 1 - turn_of : turn_of;
    const int64_t b = bh / (unsigned)a.heads, h = bh % (unsigned)a.heads;
    const int tk = (int)a.tk, i0 = (int)piece * rows_block, i1 = min(i0 + rows_block, (int)a.tq);
    const int64_t by_length = key_len ? min((int64_t)max(key_len[b], 0), a.tk) : a.tk;
    const T *s0 = s + b * a.s_b + h * a.s_h;
    T *p0 = p + b * a.p_b + h * a.p_h;
    v4u raw[kVecs];
    int seen = 0;
    auto fetch = [&](int i) {
        seen = row_seen(i, by_length, a);
#pragma unroll
        for (int v = 0; v < kVecs; ++v) raw[v] = load_slab<T, kTeam>(s0 + i * a.s_q, v * kTeam * E, me.lane, tk, seen);
    };
    int i = i0 + me.id;
    if (i < i1) fetch(i);
    for (int q = threadIdx.x; q <= bounds.n; q += kTeamBlock<kTeam>) {
        if (q < bounds.n) at[q] = bounds.at[q];
        of_bucket[q] = table[q * a.heads + h] * kLog2e;
    }
    __syncthreads();
    const int64_t first = -(int64_t)(i1 - 1) - a.offset;               // the relative position of along[0]
    for (int x = threadIdx.x; x < tk + (i1 - i0) - 1; x += kTeamBlock<kTeam>) along[x] = of_bucket[bucket_of(first + x, at, bounds.n)];
    __syncthreads();
    const float scale = a.scale * kLog2e;
    while (i < i1) {
        float t[kVecs][E], top = -INFINITY;
        const int sees = seen;
        const float *bias = along + (i1 - 1 - i);
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            const int slab = v * kTeam * E, j = slab + me.lane * E;
            if (slab >= sees) continue;
            settle_slab<T, kTeam>(raw[v], slab, me.lane, tk, tk, 0u);
            widen<T>(raw[v], t[v]);
            if (slab + kTeam * E <= sees) {
#pragma unroll
                for (int q = 0; q < E; ++q) t[v][q] = fmaf(t[v][q], scale, bias[j + q]);
            } else {
#pragma unroll
                for (int q = 0; q < E; ++q) {
                    const float f = fmaf(t[v][q], scale, bias[min(j + q, tk - 1)]);
                    t[v][q] = j + q < sees ? f : -INFINITY;
                }
            }
#pragma unroll
            for (int q = 0; q < E; ++q) top = MaxOp::apply(top, t[v][q]);
        }
        const int next = i + kTeams;
        if (next < i1) fetch(next);                                        // on its way while this row is worked on
        top = team_reduce<MaxOp, kTeam>(top, scratch);
        T *row = p0 + i * a.p_q;
        if (fabsf(top) < kPlainMax) {
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < kVecs; ++v) {
                if (v * kTeam * E >= sees) continue;
#pragma unroll
                for (int q = 0; q < E; ++q) {
                    t[v][q] = __builtin_amdgcn_exp2f(t[v][q] - top);
                    sum += t[v][q];
                }
            }
            sum = team_reduce<SumOp, kTeam>(sum, scratch2);
            float inv = __builtin_amdgcn_rcpf(sum);                        // the sum is between 1 and tk
            inv = fmaf(fmaf(-sum, inv, 1.f), inv, inv);
#pragma unroll
            for (int v = 0; v < kVecs; ++v) {
                const int slab = v * kTeam * E;
                v4u out = {0u, 0u, 0u, 0u};
                if (slab < sees) {
#pragma unroll
                    for (int q = 0; q < E; ++q) t[v][q] *= inv;
                    out = narrow<T>(t[v]);
                }
                store_slab<T, kTeam>(row, slab, me.lane, tk, out, false, a.stream_out);
            }
        } else if (sees == 0) {
#pragma unroll
            for (int v = 0; v < kVecs; ++v)
                store_slab<T, kTeam>(row, v * kTeam * E, me.lane, tk, v4u{0u, 0u, 0u, 0u}, false, a.stream_out);
            if constexpr (kTeam > kWave) __syncthreads();                  // the next row reduces in scratch again
        } else {
            // Nothing but -infinity, a NaN or a +infinity; or scores that leave fp32 in units of log 2, like a row masked
            // throughout with the type's lowest value.  In the scores' own units, from memory.
            const T *from = s0 + i * a.s_q;
            auto score = [&](int j) { return fmaf(widen1(from[j]), a.scale, bias[j] * kLn2); };
            float own = -INFINITY, sum = 0.f;
#pragma unroll 1
            for (int j = me.lane; j < sees; j += kTeam) own = MaxOp::apply(own, score(j));
            own = team_reduce<MaxOp, kTeam>(own, scratch2);
            const bool none = own == -INFINITY;
            if (!none) {
#pragma unroll 1
                for (int j = me.lane; j < sees; j += kTeam) sum += __builtin_amdgcn_exp2f((score(j) - own) * kLog2e);
            }
            sum = team_reduce<SumOp, kTeam>(sum, scratch);
            const float inv = 1.f / sum;
#pragma unroll 1
            for (int j = me.lane; j < tk; j += kTeam)
                row[j] = narrow1<T>(j < sees && !none ? __builtin_amdgcn_exp2f((score(j) - own) * kLog2e) * inv : 0.f);
            if constexpr (kTeam > kWave) __syncthreads();                  // the next row reduces in scratch again
        }
        i = next;
    }
}

// Backward: a workgroup takes `rows_block` queries of one head and sequence, each team `rows_team` (a multiple of kStep) consecutive ones.
// Of kStep rows and E keys that a lane holds, the diagonals are its registers' sums of the bucket gradient; every kStep rows they are
// added to the team's array over relative positions in LDS, in two phases because the diagonals left of a lane's first key are its
// neighbour's.  At the end the teams' arrays are added up over each bucket's positions, in a fixed order.  kBatch rows are worked on together, and as many are on their way.
template <typename T, int kTeam, int kVecs, int kStep, int kBatch>
__global__ __launch_bounds__(kTeamBlock<kTeam>) void bias_backward(T *ds, float *__restrict__ work, const T *dp, const T *__restrict__ p,
                                                                 Bounds bounds, const int32_t *__restrict__ key_len, BiasArgs a,
                                                                 int pieces, int rows_team, unsigned worker_batch)
{
    constexpr int E = kVec<T>, kThreads = kTeamBlock<kTeam>, kTeams = kThreads / kTeam, kSlots = kTeam * kVecs * E;
    static_assert(E % kStep == 0 && kStep % (2 * kBatch) == 0, "an even number of batches in a step");
    extern __shared__ float along[];                   // [teams][kSlots + rows_team - 1]; with several teams, a joined array behind
    __shared__ float scratch[2][kBatch * kThreads / kWave];
    __shared__ int32_t at[COMP_AMS_MAX_BUCKETS];
    const Team<kTeam> me;
    // with a causal mask the last queries see most: they are taken first
    const unsigned block = a.first + blockIdx.x, bh = block / (unsigned)pieces, turn_of = block % (unsigned)pieces;
    const unsigned piece = a.causal ? pieces - 1 - turn_of : turn_of;
    const unsigned b = bh / (unsigned)a.heads, h = bh % (unsigned)a.heads;
    const int tk = (int)a.tk, tq = (int)a.tq, span = kSlots + rows_team - 1;
    const int i0 = (int)piece * rows_team * kTeams, mine = i0 + me.id * rows_team, end = mine + rows_team;
    const int64_t by_length = key_len ? min((int64_t)max(key_len[b], 0), a.tk) : a.tk;
    const T *dp0 = dp + b * a.s_b + h * a.s_h, *p0 = p + b * a.p_b + h * a.p_h;
    T *ds0 = ds + b * a.o_b + h * a.o_h;
    float *diag = along + me.id * span;
    for (int q = threadIdx.x; q < bounds.n; q += kThreads) at[q] = bounds.at[q];
    for (int x = threadIdx.x; x < kTeams * span; x += kThreads) along[x] = 0.f;
    __syncthreads();
    // two batches of rows: one is worked on while the next is on its way
    v4u praw[2][kBatch][kVecs], draw[2][kBatch][kVecs];
    int seen[2][kBatch];
    auto fetch = [&](int buf, int from) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int i = from + u;
            seen[buf][u] = i < end && i < tq ? row_seen(i, by_length, a) : 0;
#pragma unroll
            for (int v = 0; v < kVecs; ++v) {
                praw[buf][u][v] = load_slab<T, kTeam>(p0 + i * a.p_q, v * kTeam * E, me.lane, tk, seen[buf][u]);
                draw[buf][u][v] = load_slab<T, kTeam>(dp0 + i * a.s_q, v * kTeam * E, me.lane, tk, seen[buf][u]);
            }
        }
    };
    fetch(0, mine);
    int turn = 0;
#pragma unroll 1
    for (int first = mine; first < end; first += kStep) {
        if (kTeam >= kWave && first >= tq) break;      // uniform over the team
        float acc[kVecs][E + kStep - 1];
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
#pragma unroll
            for (int q = 0; q < E + kStep - 1; ++q) acc[v][q] = 0.f;
#pragma unroll
        for (int batch = 0; batch < kStep; batch += kBatch) {
            constexpr int kBufs = 2;
            const int buf = batch / kBatch % kBufs;
            fetch(buf ^ 1, first + batch + kBatch);
            auto &pr = praw[buf];
            auto &dr = draw[buf];
            auto &sees = seen[buf];
            auto row_sum = [&](int u) {
                float s = 0.f;
#pragma unroll
                for (int v = 0; v < kVecs; ++v) {
                    if (v * kTeam * E < sees[u]) {
                        float pw[E], dw[E];
                        widen<T>(pr[u][v], pw);
                        widen<T>(dr[u][v], dw);
#pragma unroll
                        for (int q = 0; q < E; ++q) s = fmaf(pw[q], dw[q], s);
                    }
                }
                return s;
            };
            float total[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
#pragma unroll
                for (int v = 0; v < kVecs; ++v) {
                    if (v * kTeam * E >= sees[u]) continue;
                    settle_slab<T, kTeam>(pr[u][v], v * kTeam * E, me.lane, tk, sees[u], 0u);
                    settle_slab<T, kTeam>(dr[u][v], v * kTeam * E, me.lane, tk, tk, 0u);       // beside p = 0 it does not count
                }
                total[u] = row_sum(u);
            }
            team_reduce<SumOp, kTeam, kBatch>(total, scratch[turn]);       // the rows' reductions are independent: their steps interleave
            turn ^= 1;
            // A key of probability zero takes no gradient whatever dp holds there.  While a row's sum is of ordinary size no product was
            // NaN, so dp is finite there, dp - total too, and the formula gives zero by itself; else such keys are cleared, and looked at
            // once more below, for keys that do count may hold an infinity or a NaN.
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                if (!(fabsf(total[u]) < kPlainMax)) {
#pragma unroll
                    for (int v = 0; v < kVecs; ++v) {
                        float pw[E], dw[E];
                        widen<T>(pr[u][v], pw);
                        widen<T>(dr[u][v], dw);
#pragma unroll
                        for (int q = 0; q < E; ++q) dw[q] = pw[q] == 0.f ? 0.f : dw[q];
                        dr[u][v] = narrow<T>(dw);
                    }
                    total[u] = team_reduce<SumOp, kTeam>(row_sum(u), scratch[turn]);
                    turn ^= 1;
                }
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int i = first + batch + u;
                T *row = ds0 + i * a.o_q;
                const bool usual = fabsf(total[u]) < kPlainMax;
#pragma unroll
                for (int v = 0; v < kVecs; ++v) {
                    const int slab = v * kTeam * E;
                    v4u out = {0u, 0u, 0u, 0u};
                    if (slab < sees[u]) {
                        float pw[E], dw[E];
                        rewiden(pr[u][v]);
                        rewiden(dr[u][v]);
                        widen<T>(pr[u][v], pw);
                        widen<T>(dr[u][v], dw);
#pragma unroll
                        for (int q = 0; q < E; ++q) dw[q] = pw[q] * (dw[q] - total[u]);
                        if (!usual) {
                            asm volatile("");                  // a branch that is not taken, not a selection for every element
#pragma unroll
                            for (int q = 0; q < E; ++q) dw[q] = pw[q] == 0.f ? 0.f : dw[q];
                        }
#pragma unroll
                        for (int q = 0; q < E; ++q) {
                            acc[v][q - (batch + u) + kStep - 1] += dw[q];
                            dw[q] *= a.scale;
                        }
                        out = narrow<T>(dw);
                    }
                    if (i < tq) store_slab<T, kTeam>(row, slab, me.lane, tk, out, false, a.stream_out);
                }
            }
        }
        // diagonal a of the lane: key j0 + a seen from row `first`
        float *to = diag + (end - 1 - first) + me.lane * E;
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
#pragma unroll
            for (int q = 0; q < E; ++q) to[v * kTeam * E + q] += acc[v][q + kStep - 1];
        if constexpr (kTeam > kWave) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
#pragma unroll
            for (int q = 1; q < kStep; ++q) to[v * kTeam * E - q] += acc[v][kStep - 1 - q];
        if constexpr (kTeam > kWave) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
    __syncthreads();
    // Over the whole workgroup: place x is key x seen from its last row; team t's array begins (kTeams - 1 - t) rows_team further on.
    const int places = kSlots + kTeams * rows_team - 1;
    float *joined = kTeams > 1 ? along + kTeams * span : along;
    if constexpr (kTeams > 1) {
        for (int x = threadIdx.x; x < places; x += kThreads) {
            float s = 0.f;
#pragma unroll
            for (int t = 0; t < kTeams; ++t) {
                const int y = x - (kTeams - 1 - t) * rows_team;
                if (y >= 0 && y < span) s += along[t * span + y];
            }
            joined[x] = s;
        }
        __syncthreads();
    }
    const int64_t base = -(int64_t)(i0 + kTeams * rows_team - 1) - a.offset;      // relative position of place 0
    const unsigned w = b / worker_batch;
    const int64_t parts = (int64_t)worker_batch * pieces, part = (int64_t)(b - w * worker_batch) * pieces + piece;
    float *out = work + ((int64_t)(w * (unsigned)a.heads + h) * (bounds.n + 1)) * parts + part;
    // sixteen lanes a bucket: most buckets are narrow
    const int lane = threadIdx.x & 15;
    for (int q = threadIdx.x / 16; q <= bounds.n; q += kThreads / 16) {
        const int64_t from = q == 0 ? 0 : at[q - 1] - base, to = q == bounds.n ? places : at[q] - base;
        const int x0 = (int)min(max(from, (int64_t)0), (int64_t)places), x1 = (int)min(max(to, (int64_t)0), (int64_t)places);
        float s = 0.f;
#pragma unroll 4
        for (int x = x0 + lane; x < x1; x += 16) s += joined[x];
        s = lanes_reduce<SumOp, 16>(s);
        if (lane == 0) out[q * parts] = s;
    }
}

// work[worker][heads][buckets][parts] -> dtable[worker][buckets][heads]; one wavefront per (bucket, head, worker), lanes in a fixed
// order.
template <typename G>
__global__ __launch_bounds__(kWave) void bias_table_join(G *__restrict__ dtable, const float *__restrict__ work, int64_t heads,
                                                         int64_t parts, int buckets, int64_t grad_stride)
{
    const int64_t w = blockIdx.z, h = blockIdx.y, q = blockIdx.x;
    const float *in = work + ((w * heads + h) * buckets + q) * parts;
    float s = 0.f;
#pragma unroll 4
    for (int64_t t = threadIdx.x; t < parts; t += kWave) s += in[t];
    s = lanes_reduce<SumOp, kWave>(s);
    if (threadIdx.x == 0) dtable[w * grad_stride + q * heads + h] = narrow1<G>(s);
}

}  // namespace cams_ops
