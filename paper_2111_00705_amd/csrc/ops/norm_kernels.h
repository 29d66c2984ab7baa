// Layer norm, forward and backward, with the gradients of gain and shift reduced per worker.
//
//   mean = (1/c) sum x,  rstd = 1/sqrt((1/c) sum (x - mean)^2 + eps),  y = (x - mean) rstd gain + shift
//   xh = (x - mean) rstd,  a = dy gain:  dx = rstd (a - mean(a) - xh mean(a xh)),  dgain = sum dy xh,  dshift = sum dy
//
// HBM-bound: a row is read once and kept in registers, the variance is taken from the differences (no cancellation), and a lane keeps
// its columns' gradient sums in registers over all rows of its chunk, so that x and dy are read once for dx and both parameter
// gradients.  Measured (us of a pass among others, TB/s of what it cannot do without): forward 16384 x 768 bf16 12.2 (4.1; 50 MB, half of it in
// the memory-side cache), backward 18.9 with the join of the chunks (4.0); backward 20000 x 2047 fp32, n = 20 112 (4.4), of which the join 8.
// A copy reaches 6.1 TB/s.  One kernel per chunk of rows and a join in fixed order instead of atomics: results never vary.
#pragma once
#include "op_common.h"

namespace cams_ops {

struct NormArgs {
    int64_t rows, cols, x_stride, y_stride, dy_stride;   // y_stride: that of dx in the backward pass
    float eps, inv_cols;
    bool stream_out;                                     // y, dx are stored as a stream
};

constexpr int kNormThreads = 256;

// Rows of any length: one workgroup per row, which it reads three times (mean, variance, result).
template <typename T>
__global__ __launch_bounds__(kNormThreads) void norm_forward_any(T *y, float *__restrict__ mean, float *__restrict__ rstd,
                                                                 const T *x, const float *__restrict__ gain,
                                                                 const float *__restrict__ shift, NormArgs a)
{
    __shared__ float scratch[kNormThreads / kWave], scratch2[kNormThreads / kWave];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *xr = x + row * a.x_stride;
        T *yr = y + row * a.y_stride;
        float s = 0.f;
        for (int64_t c = threadIdx.x; c < a.cols; c += kNormThreads) s += widen1(xr[c]);
        const float mu = team_reduce<SumOp, kNormThreads>(s, scratch) * a.inv_cols;
        float q = 0.f;
        for (int64_t c = threadIdx.x; c < a.cols; c += kNormThreads) {
            const float d = widen1(xr[c]) - mu;
            q = fmaf(d, d, q);
        }
        const float r = 1.f / sqrtf(fmaf(team_reduce<SumOp, kNormThreads>(q, scratch2), a.inv_cols, a.eps));
        for (int64_t c = threadIdx.x; c < a.cols; c += kNormThreads)
            yr[c] = narrow1<T>(fmaf((widen1(xr[c]) - mu) * r, gain[c], shift ? shift[c] : 0.f));
        if (threadIdx.x == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kNormThreads) void norm_backward_any(T *dx, const T *dy, const T *x, const float *__restrict__ mean,
                                                                  const float *__restrict__ rstd, const float *__restrict__ gain,
                                                                  NormArgs a)
{
    __shared__ float scratch[kNormThreads / kWave], scratch2[kNormThreads / kWave];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *xr = x + row * a.x_stride, *dyr = dy + row * a.dy_stride;
        T *dxr = dx + row * a.y_stride;
        const float mu = mean[row], r = rstd[row];
        float s = 0.f, q = 0.f;
        for (int64_t c = threadIdx.x; c < a.cols; c += kNormThreads) {
            const float g = widen1(dyr[c]) * gain[c];
            s += g;
            q = fmaf(g, (widen1(xr[c]) - mu) * r, q);
        }
        s = team_reduce<SumOp, kNormThreads>(s, scratch) * a.inv_cols;
        q = team_reduce<SumOp, kNormThreads>(q, scratch2) * a.inv_cols;
        for (int64_t c = threadIdx.x; c < a.cols; c += kNormThreads) {
            const float xh = (widen1(xr[c]) - mu) * r;
            dxr[c] = narrow1<T>(r * (fmaf(widen1(dyr[c]), gain[c], -s) - xh * q));
        }
    }
}

// Parameter gradients of rows [chunk's rows] of one worker into work[worker][chunk][2][cols]: a workgroup takes 256 columns.
template <typename T>
__global__ __launch_bounds__(kNormThreads) void norm_param_any(float *__restrict__ work, const T *__restrict__ dy,
                                                               const T *__restrict__ x, const float *__restrict__ mean,
                                                               const float *__restrict__ rstd, NormArgs a, int64_t worker_rows,
                                                               int64_t chunk_rows)
{
    const int64_t c = (int64_t)blockIdx.x * kNormThreads + threadIdx.x;
    const int64_t lo = (int64_t)blockIdx.y * chunk_rows, hi = min(lo + chunk_rows, worker_rows);
    if (c >= a.cols) return;
    float dg = 0.f, db = 0.f;
    for (int64_t q = lo; q < hi; ++q) {
        const int64_t row = (int64_t)blockIdx.z * worker_rows + q;
        const float g = widen1(dy[row * a.dy_stride + c]);
        dg = fmaf(g, (widen1(x[row * a.x_stride + c]) - mean[row]) * rstd[row], dg);
        db += g;
    }
    float *out = work + ((int64_t)blockIdx.z * gridDim.y + blockIdx.y) * 2 * a.cols;
    out[c] = dg;
    out[a.cols + c] = db;
}

// --- rows that a team of lanes holds in registers -----------------------------------------------------------------------
//
// A team (16 lanes, a wavefront, or a workgroup) reads a row once, kVecs vectors a lane, and takes mean and variance from the
// registers; gain and shift stay in registers over the rows that a team takes in turn.

template <typename T, int kTeam, int kVecs>
__global__ __launch_bounds__(kTeamBlock<kTeam>) void norm_forward(T *y, float *__restrict__ mean, float *__restrict__ rstd, const T *x,
                                                                     const float *__restrict__ gain, const float *__restrict__ shift,
                                                                     NormArgs a)
{
    constexpr int E = kVec<T>, kTeams = kTeamBlock<kTeam> / kTeam;
    __shared__ float scratch[kTeamBlock<kTeam> / kWave], scratch2[kTeamBlock<kTeam> / kWave];
    const Team<kTeam> me;
    const int cols = (int)a.cols;
    int64_t row = (int64_t)blockIdx.x * kTeams + me.id;
    if (row >= a.rows) return;                       // a whole team; with one team per workgroup, the whole workgroup
    v4u raw[kVecs];
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int v = 0; v < kVecs; ++v) raw[v] = load_slab<T, kTeam>(x + r * a.x_stride, v * kTeam * E, me.lane, cols, cols, v < kVecs - 1);
    };
    fetch(row);
    float g[kVecs][E], b[kVecs][E];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        load_params<T, kTeam>(g[v], gain, v * kTeam * E, me.lane, cols, v < kVecs - 1);
        if (shift) {
            load_params<T, kTeam>(b[v], shift, v * kTeam * E, me.lane, cols, v < kVecs - 1);
        } else {
#pragma unroll
            for (int q = 0; q < E; ++q) b[v][q] = 0.f;
        }
    }
    for (;;) {
        float d[kVecs][E], s = 0.f;
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            settle_slab<T, kTeam>(raw[v], v * kTeam * E, me.lane, cols, cols, 0u, v < kVecs - 1);
            widen<T>(raw[v], d[v]);
#pragma unroll
            for (int q = 0; q < E; ++q) s += d[v][q];
        }
        const int64_t next = row + (int64_t)gridDim.x * kTeams;
        if (next < a.rows) fetch(next);              // on its way while this row is worked on
        const float mu = team_reduce<SumOp, kTeam>(s, scratch) * a.inv_cols;
        float var = 0.f;
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            const int at = v * kTeam * E + me.lane * E;
#pragma unroll
            for (int q = 0; q < E; ++q) d[v][q] -= mu;
            if (v < kVecs - 1 || (v + 1) * kTeam * E <= cols) {
#pragma unroll
                for (int q = 0; q < E; ++q) var = fmaf(d[v][q], d[v][q], var);
            } else {
#pragma unroll
                for (int q = 0; q < E; ++q)
                    if (at + q < cols) var = fmaf(d[v][q], d[v][q], var);
            }
        }
        const float r = 1.f / sqrtf(fmaf(team_reduce<SumOp, kTeam>(var, scratch2), a.inv_cols, a.eps));
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
#pragma unroll
            for (int q = 0; q < E; ++q) d[v][q] = fmaf(d[v][q] * r, g[v][q], b[v][q]);
            store_slab<T, kTeam>(y + row * a.y_stride, v * kTeam * E, me.lane, cols, narrow<T>(d[v]), v < kVecs - 1, a.stream_out);
        }
        if (me.lane == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
        if (next >= a.rows) return;
        row = next;
    }
}

// Backward: the rows of one chunk of one worker, the teams in turn; every lane adds up the parameter gradients of its columns over
// its rows, the teams' sums are joined in order, and work[worker][chunk] receives 2 x cols of them.
template <typename T, int kTeam, int kVecs>
__global__ __launch_bounds__(kTeamBlock<kTeam>) void norm_backward(T *dx, float *__restrict__ work, const T *dy, const T *x,
                                                                      const float *__restrict__ mean, const float *__restrict__ rstd,
                                                                      const float *__restrict__ gain, NormArgs a, int64_t worker_rows,
                                                                      int64_t chunk_rows)
{
    constexpr int E = kVec<T>, kTeams = kTeamBlock<kTeam> / kTeam, kSlots = kTeam * kVecs * E;
    __shared__ float scratch[2][2 * kTeamBlock<kTeam> / kWave];
    __shared__ float joined[kTeams > 1 ? kTeams * kSlots : 1];
    const Team<kTeam> me;
    const int cols = (int)a.cols;
    const int64_t base = (int64_t)blockIdx.y * worker_rows;
    const int64_t lo = base + (int64_t)blockIdx.x * chunk_rows, hi = base + min(((int64_t)blockIdx.x + 1) * chunk_rows, worker_rows);
    float g[kVecs][E], dg[kVecs][E], db[kVecs][E];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        load_params<T, kTeam>(g[v], gain, v * kTeam * E, me.lane, cols, v < kVecs - 1);
#pragma unroll
        for (int q = 0; q < E; ++q) dg[v][q] = db[v][q] = 0.f;
    }
    v4u xraw[kVecs], dyraw[kVecs];
    float mu = 0.f, r = 0.f;
    auto fetch = [&](int64_t at) {
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            xraw[v] = load_slab<T, kTeam>(x + at * a.x_stride, v * kTeam * E, me.lane, cols, cols, v < kVecs - 1);
            dyraw[v] = load_slab<T, kTeam>(dy + at * a.dy_stride, v * kTeam * E, me.lane, cols, cols, v < kVecs - 1);
        }
        mu = mean[at];
        r = rstd[at];
    };
    int64_t row = lo + me.id;
    int turn = 0;
    if (row < hi) fetch(row);
    while (row < hi) {
        float xh[kVecs][E], up[kVecs][E], sums[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            settle_slab<T, kTeam>(xraw[v], v * kTeam * E, me.lane, cols, cols, 0u, v < kVecs - 1);
            settle_slab<T, kTeam>(dyraw[v], v * kTeam * E, me.lane, cols, cols, 0u, v < kVecs - 1);
            widen<T>(xraw[v], xh[v]);
            widen<T>(dyraw[v], up[v]);
#pragma unroll
            for (int q = 0; q < E; ++q) {
                xh[v][q] = (xh[v][q] - mu) * r;        // past the row: finite, times a zero gradient
                const float t = up[v][q] * g[v][q];
                sums[0] += t;
                sums[1] = fmaf(t, xh[v][q], sums[1]);
                dg[v][q] = fmaf(up[v][q], xh[v][q], dg[v][q]);
                db[v][q] += up[v][q];
            }
        }
        const float scale = r;
        const int64_t next = row + kTeams;
        if (next < hi) fetch(next);
        team_reduce<SumOp, kTeam, 2>(sums, scratch[turn]);
        turn ^= 1;
        const float s = sums[0] * a.inv_cols, q2 = sums[1] * a.inv_cols;
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
#pragma unroll
            for (int q = 0; q < E; ++q) up[v][q] = scale * (fmaf(up[v][q], g[v][q], -s) - xh[v][q] * q2);
            store_slab<T, kTeam>(dx + row * a.y_stride, v * kTeam * E, me.lane, cols, narrow<T>(up[v]), v < kVecs - 1, a.stream_out);
        }
        row = next;
    }
    float *out = work + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * a.cols;
    auto emit = [&](float (&acc)[kVecs][E], float *to) {
        if constexpr (kTeams == 1) {
#pragma unroll
            for (int v = 0; v < kVecs; ++v)
#pragma unroll
                for (int q = 0; q < E; ++q) {
                    const int c = v * kTeam * E + me.lane * E + q;
                    if (c < cols) to[c] = acc[v][q];
                }
        } else {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < kVecs; ++v)
#pragma unroll
                for (int q = 0; q < E; ++q) joined[me.id * kSlots + v * kTeam * E + me.lane * E + q] = acc[v][q];
            __syncthreads();
            for (int c = threadIdx.x; c < cols; c += kTeamBlock<kTeam>) {
                float sum = joined[c];
#pragma unroll
                for (int t = 1; t < kTeams; ++t) sum += joined[t * kSlots + c];
                to[c] = sum;
            }
        }
    };
    emit(dg, out);
    emit(db, out + a.cols);
}

// The chunks' sums into the workers' rows of gradients: 32 columns a workgroup, eight lanes a column that take every eighth chunk
// in ascending order and are then added in order.
constexpr int kJoinCols = 32, kJoinParts = kNormThreads / kJoinCols;
template <typename G>
__global__ __launch_bounds__(kNormThreads) void norm_param_join(G *__restrict__ dgain, G *__restrict__ dshift,
                                                                const float *__restrict__ work, int64_t cols, int chunks,
                                                                int64_t grad_stride, unsigned first)
{
    __shared__ float parts[kJoinParts][kJoinCols];
    const int part = threadIdx.x / kJoinCols, lane = threadIdx.x % kJoinCols;
    const int64_t c = (int64_t)(first + blockIdx.x) * kJoinCols + lane;
    float s = 0.f;
    if (c < 2 * cols) {
        const float *in = work + (int64_t)blockIdx.y * chunks * 2 * cols + c;
#pragma unroll 8
        for (int q = part; q < chunks; q += kJoinParts) s += in[(int64_t)q * 2 * cols];
    }
    parts[part][lane] = s;
    __syncthreads();
    if (part != 0 || c >= 2 * cols) return;
#pragma unroll
    for (int q = 1; q < kJoinParts; ++q) s += parts[q][lane];
    const int64_t at = (int64_t)blockIdx.y * grad_stride;
    if (c < cols) dgain[at + c] = narrow1<G>(s);
    else if (dshift) dshift[at + c - cols] = narrow1<G>(s);
}

}  // namespace cams_ops
