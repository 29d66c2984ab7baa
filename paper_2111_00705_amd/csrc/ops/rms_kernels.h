// Root-mean-square norm with the residual's addition, forward (in the activations' type, or in 8 bits) and backward with the gain's
// gradients reduced per worker.
//
//   h = x + residual, rounded to the type;  rstd = 1/sqrt((1/c) sum h^2 + eps);  y = h rstd gain
//   xh = h rstd,  a = dy gain:  dx = rstd (a - xh mean(a xh)) + dresidual,  dgain = sum dy xh
//
// HBM-bound: a row is read once and kept in registers, where it is added, normed and rounded; the next row is on its way meanwhile.  A
// lane keeps its columns' gradient sums in registers over all rows of its chunk, as in norm_kernels.h.
// Measured alone, with TB/s of what has to move: forward in 8 bits 16384 x 2048 bf16 with residual 39.6 us (235 MB, 5.9); backward 16384 x 768
// bf16, n = 8 18.4 (101 MB, 5.5) and 4.0 for the join of its chunks; 20000 x 2047 fp32 kept in 8 bits, n = 20 87 to 107 (533 MB, 5.0 to 6.1: rows of
// odd length, one in flight a workgroup beside the one worked on).  A copy reaches 6.1 TB/s.
#pragma once
#include "rows8.h"

namespace cams_ops {

struct RmsArgs {
    int64_t rows, cols, x_stride, r_stride, h_stride, y_stride;
    float eps, inv_cols;
    bool binary, stream_in, stream_out, stream_h;      // x and residual, y, h pass the caches by
};

constexpr int kRmsThreads = 256;

// x + residual as the type holds it: what the norm is of is what the backward pass will read.
template <typename T> __device__ __forceinline__ float rounded(float x) { return widen1(narrow1<T>(x)); }

// Rows of any length: a workgroup a row, which it reads two or three times.  h is written last: it may replace x or the residual.
template <typename T, bool kQ8>
__global__ __launch_bounds__(kRmsThreads) void rms_forward_any(void *y, float *__restrict__ scale, T *h, float *__restrict__ rstd, const T *x,
                                                               const T *residual, const float *__restrict__ gain, RmsArgs a)
{
    __shared__ float scratch[kRmsThreads / kWave], scratch2[kRmsThreads / kWave];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *xr = x + row * a.x_stride, *rr = residual ? residual + row * a.r_stride : nullptr;
        auto at = [&](int64_t c) {
            const float v = widen1(xr[c]);
            return rr ? rounded<T>(v + widen1(rr[c])) : v;
        };
        float s = 0.f;
        for (int64_t c = threadIdx.x; c < a.cols; c += kRmsThreads) s = fmaf(at(c), at(c), s);
        const float r = 1.f / sqrtf(fmaf(team_reduce<SumOp, kRmsThreads>(s, scratch), a.inv_cols, a.eps));
        RowScale rs = {0.f, 0.f, 0.f};
        if constexpr (kQ8) {
            float top = 0.f;
            for (int64_t c = threadIdx.x; c < a.cols; c += kRmsThreads) top = MaxOp::apply(top, fabsf(at(c) * r * gain[c]));
            rs = row_scale(team_reduce<MaxOp, kRmsThreads>(top, scratch2), a.binary, kFiniteMax<float>);
        } else {
            __syncthreads();                         // before the scratch of the next row
        }
        for (int64_t c = threadIdx.x; c < a.cols; c += kRmsThreads) {
            const float v = at(c), out = v * r * gain[c];
            if constexpr (kQ8) static_cast<int8_t *>(y)[row * a.y_stride + c] = (int8_t)byte_of(out, rs);
            else static_cast<T *>(y)[row * a.y_stride + c] = narrow1<T>(out);
            if (h) h[row * a.h_stride + c] = narrow1<T>(v);
        }
        if (threadIdx.x == 0) {
            if (rstd) rstd[row] = r;
            if constexpr (kQ8) scale[row] = rs.scale;
        }
    }
}

// Rows that a team of lanes holds in registers.
template <typename T, int kTeam, int kVecs, bool kQ8>
__global__ __launch_bounds__(kTeamBlock<kTeam>) void rms_forward(void *y, float *__restrict__ scale, T *h, float *__restrict__ rstd, const T *x,
                                                                 const T *residual, const float *__restrict__ gain, RmsArgs a)
{
    constexpr int E = kVec<T>, kTeams = kTeamBlock<kTeam> / kTeam;
    __shared__ float scratch[kTeamBlock<kTeam> / kWave], scratch2[kTeamBlock<kTeam> / kWave];
    const Team<kTeam> me;
    const int cols = (int)a.cols;
    int64_t row = (int64_t)blockIdx.x * kTeams + me.id;
    if (row >= a.rows) return;                       // a whole team; with one team per workgroup, the whole workgroup
    v4u xraw[kVecs], rraw[kVecs];
    auto fetch = [&](int64_t at) {
#pragma unroll
        for (int v = 0; v < kVecs; ++v) xraw[v] = load_slab<T, kTeam>(x + at * a.x_stride, v * kTeam * E, me.lane, cols, cols, v < kVecs - 1, a.stream_in);
        if (residual) {
#pragma unroll
            for (int v = 0; v < kVecs; ++v)
                rraw[v] = load_slab<T, kTeam>(residual + at * a.r_stride, v * kTeam * E, me.lane, cols, cols, v < kVecs - 1, a.stream_in);
        }
    };
    fetch(row);
    float g[kVecs][E];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) load_params<T, kTeam>(g[v], gain, v * kTeam * E, me.lane, cols, v < kVecs - 1);
    for (;;) {
        float d[kVecs][E], s = 0.f;
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            settle_slab<T, kTeam>(xraw[v], v * kTeam * E, me.lane, cols, cols, 0u, v < kVecs - 1);
            if (residual) {
                float w[E], u[E];
                settle_slab<T, kTeam>(rraw[v], v * kTeam * E, me.lane, cols, cols, 0u, v < kVecs - 1);
                widen<T>(xraw[v], w);
                widen<T>(rraw[v], u);
#pragma unroll
                for (int q = 0; q < E; ++q) w[q] += u[q];
                xraw[v] = narrow<T>(w);
            }
            if (h) store_slab<T, kTeam>(h + row * a.h_stride, v * kTeam * E, me.lane, cols, xraw[v], v < kVecs - 1, a.stream_h);
            widen<T>(xraw[v], d[v]);
#pragma unroll
            for (int q = 0; q < E; ++q) s = fmaf(d[v][q], d[v][q], s);
        }
        const int64_t next = row + (int64_t)gridDim.x * kTeams;
        if (next < a.rows) fetch(next);              // on its way while this row is worked on
        const float r = 1.f / sqrtf(fmaf(team_reduce<SumOp, kTeam>(s, scratch), a.inv_cols, a.eps));
        float top = 0.f;
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
#pragma unroll
            for (int q = 0; q < E; ++q) {
                d[v][q] = d[v][q] * r * g[v][q];
                if constexpr (kQ8) top = MaxOp::apply(top, fabsf(d[v][q]));
            }
            if constexpr (!kQ8)
                store_slab<T, kTeam>(static_cast<T *>(y) + row * a.y_stride, v * kTeam * E, me.lane, cols, narrow<T>(d[v]), v < kVecs - 1,
                                     a.stream_out);
        }
        if constexpr (kQ8) {
            const RowScale rs = row_scale(team_reduce<MaxOp, kTeam>(top, scratch2), a.binary, kFiniteMax<float>);
#pragma unroll
            for (int v = 0; v < kVecs; ++v)
                store_byte_slab<E, kTeam>(static_cast<int8_t *>(y) + row * a.y_stride, v * kTeam * E, me.lane, cols, bytes_of<E>(d[v], rs),
                                          v < kVecs - 1);
            if (me.lane == 0) scale[row] = rs.scale;
        } else if constexpr (kTeam > kWave) {
            __syncthreads();                         // before the scratch of the next row
        }
        if (me.lane == 0 && rstd) rstd[row] = r;
        if (next >= a.rows) return;
        row = next;
    }
}

struct RmsBackArgs {
    int64_t rows, cols, dx_stride, dy_stride, h_stride, r_stride;
    float inv_cols;
    bool stream_in, stream_out;
    void *dgain;                 // where a worker's rows are one chunk, its sums go there at once, in the gradients' type
    int64_t grad_stride;
    int grad_type;               // 0: fp32, 1: bfloat16, 2: half precision
};

// The kept row is in the gradients' type, or in 8 bits with a scale.
template <typename H> constexpr bool kKept8 = sizeof(H) == 1;

template <typename T, typename H>
__global__ __launch_bounds__(kRmsThreads) void rms_backward_any(T *dx, const T *dy, const H *h, const float *__restrict__ h_scale,
                                                                const float *__restrict__ rstd, const float *__restrict__ gain,
                                                                const T *dresidual, RmsBackArgs a)
{
    __shared__ float scratch[2][kRmsThreads / kWave];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const H *hr = h + row * a.h_stride;
        const T *dyr = dy + row * a.dy_stride;
        const float r = rstd[row];
        auto unit = [&](int64_t c) {
            if constexpr (kKept8<H>) return (float)hr[c] * h_scale[row] * r;
            else return widen1(hr[c]) * r;
        };
        float s = 0.f;
        for (int64_t c = threadIdx.x; c < a.cols; c += kRmsThreads) s = fmaf(widen1(dyr[c]) * gain[c], unit(c), s);
        s = team_reduce<SumOp, kRmsThreads>(s, scratch[turn]) * a.inv_cols;
        for (int64_t c = threadIdx.x; c < a.cols; c += kRmsThreads) {
            float d = r * (widen1(dyr[c]) * gain[c] - unit(c) * s);
            if (dresidual) d += widen1(dresidual[row * a.r_stride + c]);
            dx[row * a.dx_stride + c] = narrow1<T>(d);
        }
    }
}

// The gain's gradients of the rows of a chunk of a worker into work[worker][chunk][cols]: a workgroup takes 256 columns.
template <typename T, typename H>
__global__ __launch_bounds__(kRmsThreads) void rms_param_any(float *__restrict__ work, const T *__restrict__ dy, const H *__restrict__ h,
                                                             const float *__restrict__ h_scale, const float *__restrict__ rstd,
                                                             RmsBackArgs a, int64_t worker_rows, int64_t chunk_rows, unsigned first)
{
    const int64_t c = (int64_t)(first + blockIdx.x) * kRmsThreads + threadIdx.x;
    const int64_t lo = (int64_t)blockIdx.y * chunk_rows, hi = min(lo + chunk_rows, worker_rows);
    if (c >= a.cols) return;
    float dg = 0.f;
    for (int64_t q = lo; q < hi; ++q) {
        const int64_t row = (int64_t)blockIdx.z * worker_rows + q;
        float xh;
        if constexpr (kKept8<H>) xh = (float)h[row * a.h_stride + c] * h_scale[row] * rstd[row];
        else xh = widen1(h[row * a.h_stride + c]) * rstd[row];
        dg = fmaf(widen1(dy[row * a.dy_stride + c]), xh, dg);
    }
    work[((int64_t)blockIdx.z * gridDim.y + blockIdx.y) * a.cols + c] = dg;
}

// The rows of one chunk of one worker, the teams in turn; every lane adds up the gain's gradients of its columns over its rows, the
// teams' sums are joined in order, and work[worker][chunk] receives them.
template <typename T, typename H, int kTeam, int kVecs>
__global__ __launch_bounds__(kTeamBlock<kTeam>) void rms_backward(T *dx, float *__restrict__ work, const T *dy, const H *h,
                                                                  const float *__restrict__ h_scale, const float *__restrict__ rstd,
                                                                  const float *__restrict__ gain, const T *dresidual, RmsBackArgs a,
                                                                  int64_t worker_rows, int64_t chunk_rows)
{
    constexpr int E = kVec<T>, kTeams = kTeamBlock<kTeam> / kTeam, kSlots = kTeam * kVecs * E;
    constexpr bool k8 = kKept8<H>;
    __shared__ float scratch[2][kTeamBlock<kTeam> / kWave];
    __shared__ float joined[kTeams > 1 ? kTeams * kSlots : 1];
    const Team<kTeam> me;
    const int cols = (int)a.cols;
    const int64_t base = (int64_t)blockIdx.y * worker_rows;
    const int64_t lo = base + (int64_t)blockIdx.x * chunk_rows, hi = base + min(((int64_t)blockIdx.x + 1) * chunk_rows, worker_rows);
    float g[kVecs][E], dg[kVecs][E];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        load_params<T, kTeam>(g[v], gain, v * kTeam * E, me.lane, cols, v < kVecs - 1);
#pragma unroll
        for (int q = 0; q < E; ++q) dg[v][q] = 0.f;
    }
    v4u hraw[kVecs], dyraw[kVecs], rraw[kVecs];
    uint64_t h8[kVecs];
    float r = 0.f, hs = 0.f;
    auto fetch = [&](int64_t at) {
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            if constexpr (k8) h8[v] = load_byte_slab<E, kTeam>(h + at * a.h_stride, v * kTeam * E, me.lane, cols, v < kVecs - 1);
            else hraw[v] = load_slab<T, kTeam>(h + at * a.h_stride, v * kTeam * E, me.lane, cols, cols, v < kVecs - 1, a.stream_in);
            dyraw[v] = load_slab<T, kTeam>(dy + at * a.dy_stride, v * kTeam * E, me.lane, cols, cols, v < kVecs - 1, a.stream_in);
        }
        if (dresidual) {
#pragma unroll
            for (int v = 0; v < kVecs; ++v)
                rraw[v] = load_slab<T, kTeam>(dresidual + at * a.r_stride, v * kTeam * E, me.lane, cols, cols, v < kVecs - 1, a.stream_in);
        }
        r = rstd[at];
        if constexpr (k8) hs = h_scale[at];
    };
    int64_t row = lo + me.id;
    int turn = 0;
    if (row < hi) fetch(row);
    while (row < hi) {
        float xh[kVecs][E], up[kVecs][E], s = 0.f;
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            settle_slab<T, kTeam>(dyraw[v], v * kTeam * E, me.lane, cols, cols, 0u, v < kVecs - 1);
            widen<T>(dyraw[v], up[v]);
            if constexpr (k8) {
                settle_bytes<E, kTeam>(h8[v], v * kTeam * E, me.lane, cols, v < kVecs - 1);
                from_bytes<E>(h8[v], xh[v]);
#pragma unroll
                for (int q = 0; q < E; ++q) xh[v][q] *= hs;
            } else {
                settle_slab<T, kTeam>(hraw[v], v * kTeam * E, me.lane, cols, cols, 0u, v < kVecs - 1);
                widen<T>(hraw[v], xh[v]);
            }
#pragma unroll
            for (int q = 0; q < E; ++q) {
                xh[v][q] *= r;
                dg[v][q] = fmaf(up[v][q], xh[v][q], dg[v][q]);
                up[v][q] *= g[v][q];
                s = fmaf(up[v][q], xh[v][q], s);
            }
        }
        if (dresidual) {
#pragma unroll
            for (int v = 0; v < kVecs; ++v) {
                settle_slab<T, kTeam>(rraw[v], v * kTeam * E, me.lane, cols, cols, 0u, v < kVecs - 1);
                rewiden(rraw[v]);                    // it has arrived before another wavefront's dx may replace it
            }
        }
        const float mean = team_reduce<SumOp, kTeam>(s, scratch[turn]) * a.inv_cols;
        turn ^= 1;
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
#pragma unroll
            for (int q = 0; q < E; ++q) up[v][q] = r * (up[v][q] - xh[v][q] * mean);
            if (dresidual) {
                float w[E];
                widen<T>(rraw[v], w);
#pragma unroll
                for (int q = 0; q < E; ++q) up[v][q] += w[q];
            }
            dyraw[v] = narrow<T>(up[v]);
        }
        const int64_t now = row;
        row += kTeams;
        v4u out[kVecs];
#pragma unroll
        for (int v = 0; v < kVecs; ++v) out[v] = dyraw[v];
        if (row < hi) fetch(row);
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
            store_slab<T, kTeam>(dx + now * a.dx_stride, v * kTeam * E, me.lane, cols, out[v], v < kVecs - 1, a.stream_out);
    }
    float *to = work + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * a.cols;
    const bool only = gridDim.x == 1;
    auto emit = [&](int c, float sum) {
        if (!only) {
            to[c] = sum;
            return;
        }
        const int64_t at = (int64_t)blockIdx.y * a.grad_stride + c;
        if (a.grad_type == 0) static_cast<float *>(a.dgain)[at] = sum;
        else if (a.grad_type == 1) static_cast<bf16_t *>(a.dgain)[at] = narrow1<bf16_t>(sum);
        else static_cast<f16_t *>(a.dgain)[at] = narrow1<f16_t>(sum);
    };
    if constexpr (kTeams == 1) {
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
#pragma unroll
            for (int q = 0; q < E; ++q) {
                const int c = v * kTeam * E + me.lane * E + q;
                if (c < cols) emit(c, dg[v][q]);
            }
    } else {
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
#pragma unroll
            for (int q = 0; q < E; ++q) joined[me.id * kSlots + v * kTeam * E + me.lane * E + q] = dg[v][q];
        __syncthreads();
        for (int c = threadIdx.x; c < cols; c += kTeamBlock<kTeam>) {
            float sum = joined[c];
#pragma unroll
            for (int t = 1; t < kTeams; ++t) sum += joined[t * kSlots + c];
            emit(c, sum);
        }
    }
}

// Chunks' sums work[worker][chunk][cols] into the workers' rows of gradients: 32 columns a workgroup, eight lanes a column that take
// every eighth chunk in ascending order and are then added in order.
constexpr int kColumnsJoin = 32, kColumnsParts = kRmsThreads / kColumnsJoin;
template <typename G>
__global__ __launch_bounds__(kRmsThreads) void columns_join(G *__restrict__ grad, const float *__restrict__ work, int64_t cols, int chunks,
                                                            int64_t grad_stride, unsigned first)
{
    __shared__ float parts[kColumnsParts][kColumnsJoin];
    const int part = threadIdx.x / kColumnsJoin, lane = threadIdx.x % kColumnsJoin;
    const int64_t c = (int64_t)(first + blockIdx.x) * kColumnsJoin + lane;
    float s = 0.f;
    if (c < cols) {
        const float *in = work + (int64_t)blockIdx.y * chunks * cols + c;
#pragma unroll 8
        for (int q = part; q < chunks; q += kColumnsParts) s += in[(int64_t)q * cols];
    }
    parts[part][lane] = s;
    __syncthreads();
    if (part != 0 || c >= cols) return;
#pragma unroll
    for (int q = 1; q < kColumnsParts; ++q) s += parts[q][lane];
    grad[(int64_t)blockIdx.y * grad_stride + c] = narrow1<G>(s);
}

}  // namespace cams_ops
