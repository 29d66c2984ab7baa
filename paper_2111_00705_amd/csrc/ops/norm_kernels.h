// Layer norm, forward and backward, with the gradients of gain and shift reduced per worker.
#pragma once
#include "op_common.h"

namespace cams_ops {

struct NormArgs {
    int64_t rows, cols, x_stride, y_stride, dy_stride;   // y_stride: that of dx in the backward pass
    float eps, inv_cols;
};

constexpr int kNormThreads = 256;

// Rows of any length: one workgroup per row, which it reads three times (mean, variance, result).
template <typename T>
__global__ __launch_bounds__(kNormThreads) void norm_forward_any(T *y, float *__restrict__ mean, float *__restrict__ rstd,
                                                                 const T *x, const float *__restrict__ gain,
                                                                 const float *__restrict__ shift, NormArgs a)
{
    __shared__ float scratch[kNormThreads / kWave];
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
        const float r = 1.f / sqrtf(fmaf(team_reduce<SumOp, kNormThreads>(q, scratch), a.inv_cols, a.eps));
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
    __shared__ float scratch[kNormThreads / kWave];
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
        q = team_reduce<SumOp, kNormThreads>(q, scratch) * a.inv_cols;
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

// The chunks' sums, added in ascending order, into the workers' rows of gradients.
template <typename G>
__global__ __launch_bounds__(kNormThreads) void norm_param_join(G *__restrict__ dgain, G *__restrict__ dshift,
                                                                const float *__restrict__ work, int64_t cols, int chunks,
                                                                int64_t grad_stride)
{
    const int64_t c = (int64_t)blockIdx.x * kNormThreads + threadIdx.x;
    if (c >= 2 * cols) return;
    const float *in = work + (int64_t)blockIdx.y * chunks * 2 * cols + c;
    float s = 0.f;
    for (int q = 0; q < chunks; ++q) s += in[(int64_t)q * 2 * cols];
    const int64_t at = (int64_t)blockIdx.y * grad_stride;
    if (c < cols) dgain[at + c] = narrow1<G>(s);
    else if (dshift) dshift[at + c - cols] = narrow1<G>(s);
}

}  // namespace cams_ops
