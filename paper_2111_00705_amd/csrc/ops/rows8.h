// Rows held in 8 bits: q int8, one fp32 scale a row, x ~ q scale.
//
//   scale = max(absmax / 127, 2^-126), or the least power of two not below that;  q = rint(x (1 / scale)), |q| <= 127
//
// A row's values are read, reduced to their largest magnitude and rounded while they stand in registers.  Scales that are powers of two
// make every product q scale a number of 7 bits: restored values are exact in any of the types, and so are the products of a backward
// pass that reads the row (weight_kernels.h); the price is up to one bit, half a bit on average.
//
// HBM-bound: a row is read once and written once.  16384 x 4096 bf16: to 8 bits 29.6 us (201 MB, 6.8 TB/s), back 28.8 (7.0; the 8 bits come from the
// memory-side cache).  Teams of 16 lanes to a workgroup of 1024 hold a row in registers between its maximum and its rounding, so that no second
// read is needed up to 32768 elements of 16 bits, 16384 of 32.
#pragma once
#include "op_common.h"

namespace cams_ops {

// The largest fp32 number that rounds to a finite one of the type: what is restored from a row stays finite where the row was.
template <typename T> constexpr float kFiniteMax = 0x1.fffffep+127f;
template <> constexpr float kFiniteMax<bf16_t> = 0x1.fefffep+127f;      // below 2^128 (1 - 2^-9)
template <> constexpr float kFiniteMax<f16_t> = 0x1.ffdffep+15f;          // below 65520

struct RowScale {
    float scale, inv, most;      // most: largest |q|
};

// A row with a NaN or an infinity has the scale NaN and zeros in q: it is restored as NaN.
__device__ __forceinline__ RowScale row_scale(float absmax, bool binary, float finite_max)
{
    if (!(absmax < INFINITY)) return {NAN, 0.f, 0.f};
    float s = fmaxf(absmax / 127.f, 0x1p-126f);
    if (binary) s = __uint_as_float((__float_as_uint(s) + 0x7fffffu) & 0x7f800000u);
    const float most = 127.f * s <= finite_max ? 127.f : fminf(126.f, floorf(finite_max / s));
    return {s, 1.f / s, most};
}

// The 8 bits of rint(x inv), in the low byte: product and addition are rounded one after the other, the addition of 1.5 2^23 to whole
// numbers, ties to even.  A NaN comes out as -most, which is zero where a row has one.
__device__ __forceinline__ uint32_t byte_of(float x, const RowScale &r)
{
    return __float_as_uint(__builtin_amdgcn_fmed3f(x * r.inv, -r.most, r.most) + 12582912.f);
}

// Four bytes in order.
__device__ __forceinline__ uint32_t four_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), hi = __builtin_amdgcn_perm(d, c, 0x0c0c0400u);
    return lo | (hi << 16);
}

template <int E> __device__ __forceinline__ uint64_t bytes_of(const float (&x)[E], const RowScale &r)
{
    uint64_t raw = four_bytes(byte_of(x[0], r), byte_of(x[1], r), byte_of(x[2], r), byte_of(x[3], r));
    if constexpr (E == 8) raw |= (uint64_t)four_bytes(byte_of(x[4], r), byte_of(x[5], r), byte_of(x[6], r), byte_of(x[7], r)) << 32;
    return raw;
}

template <int E> __device__ __forceinline__ void from_bytes(uint64_t raw, float (&x)[E])
{
#pragma unroll
    for (int q = 0; q < E; ++q) x[q] = (float)(int8_t)(raw >> (8 * q));
}

typedef uint32_t u32_1 __attribute__((aligned(1)));
typedef uint16_t u16_1 __attribute__((aligned(1)));
typedef uint32_t v2u_1 __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t v4u_1 __attribute__((ext_vector_type(4), aligned(1)));

template <int E> __device__ __forceinline__ uint64_t load_bytes(const int8_t *p)
{
    if constexpr (E == 4) return *reinterpret_cast<const u32_1 *>(p);
    const v2u_1 v = *reinterpret_cast<const v2u_1 *>(p);
    return ((uint64_t)v[1] << 32) | v[0];
}

// The bytes of a lane's E elements in slabs as in op_common.h: those past the row are zero.  The row has at least E elements.
// Where the row ends inside, its last E bytes are loaded; settle_bytes moves them into place.
template <int E, int kTeam>
__device__ __forceinline__ uint64_t load_byte_slab(const int8_t *row, int first, int lane, int len, bool sure)
{
    const int at = first + lane * E;
    if (sure || first + kTeam * E <= len) return load_bytes<E>(row + at);
    return at < len ? load_bytes<E>(row + min(at, len - E)) : 0;
}
template <int E, int kTeam>
__device__ __forceinline__ void settle_bytes(uint64_t &raw, int first, int lane, int len, bool sure)
{
    if (sure || first + kTeam * E <= len) return;
    const int late = first + lane * E - (len - E);
    if (late > 0) raw = late < E ? raw >> (8 * late) : 0;
}
template <int E, int kTeam>
__device__ __forceinline__ void store_byte_slab(int8_t *row, int first, int lane, int len, uint64_t raw, bool sure)
{
    const int at = first + lane * E;
    int8_t *p = row + at;
    if (sure || first + kTeam * E <= len || at + E <= len) {
        if constexpr (E == 4) *reinterpret_cast<u32_1 *>(p) = (uint32_t)raw;
        else *reinterpret_cast<v2u_1 *>(p) = v2u_1{(uint32_t)raw, (uint32_t)(raw >> 32)};
    } else if (at < len) {                          // a binary number of elements is left
        const int rest = len - at;
        if (E == 8 && (rest & 4)) {
            *reinterpret_cast<u32_1 *>(p) = (uint32_t)raw;
            raw >>= 32;
            p += 4;
        }
        if (rest & 2) {
            *reinterpret_cast<u16_1 *>(p) = (uint16_t)raw;
            raw >>= 16;
            p += 2;
        }
        if (rest & 1) *p = (int8_t)raw;
    }
}

struct QuantArgs {
    int64_t rows, cols, x_stride, q_stride;
    bool binary, stream;         // stream: the wide rows pass the caches by
    int64_t first;               // workgroups of the launches before
};

constexpr int kQuantThreads = 256;

// Rows of any length: a workgroup a row, which it reads twice.
template <typename T>
__global__ __launch_bounds__(kQuantThreads) void quantize_any(int8_t *__restrict__ q, float *__restrict__ scale, const T *__restrict__ x, QuantArgs a)
{
    __shared__ float scratch[2][kQuantThreads / kWave];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const T *xr = x + row * a.x_stride;
        float top = 0.f;
        for (int64_t c = threadIdx.x; c < a.cols; c += kQuantThreads) top = MaxOp::apply(top, fabsf(widen1(xr[c])));
        const RowScale r = row_scale(team_reduce<MaxOp, kQuantThreads>(top, scratch[turn]), a.binary, kFiniteMax<T>);
        for (int64_t c = threadIdx.x; c < a.cols; c += kQuantThreads) q[row * a.q_stride + c] = (int8_t)byte_of(widen1(xr[c]), r);
        if (threadIdx.x == 0) scale[row] = r.scale;
    }
}

template <typename T>
__global__ __launch_bounds__(kQuantThreads) void restore_any(T *__restrict__ x, const int8_t *__restrict__ q, const float *__restrict__ scale,
                                                             QuantArgs a)
{
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float s = scale[row];
        for (int64_t c = threadIdx.x; c < a.cols; c += kQuantThreads) x[row * a.x_stride + c] = narrow1<T>((float)q[row * a.q_stride + c] * s);
    }
}

// Rows that a team of lanes holds in registers: read once, written once.
template <typename T, int kTeam, int kVecs>
__global__ __launch_bounds__(kTeamBlock<kTeam>) void quantize(int8_t *__restrict__ q, float *__restrict__ scale, const T *__restrict__ x, QuantArgs a)
{
    constexpr int E = kVec<T>, kTeams = kTeamBlock<kTeam> / kTeam;
    __shared__ float scratch[kTeamBlock<kTeam> / kWave];
    const Team<kTeam> me;
    const int cols = (int)a.cols;
    const int64_t row = (a.first + blockIdx.x) * kTeams + me.id;
    if (row >= a.rows) return;                       // a whole team; with one team per workgroup, the whole workgroup
    v4u raw[kVecs];
#pragma unroll
    for (int v = 0; v < kVecs; ++v)
        raw[v] = load_slab<T, kTeam>(x + row * a.x_stride, v * kTeam * E, me.lane, cols, cols, v < kVecs - 1, a.stream);
    float top = 0.f;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        settle_slab<T, kTeam>(raw[v], v * kTeam * E, me.lane, cols, cols, 0u, v < kVecs - 1);
        float w[E];
        widen<T>(raw[v], w);
#pragma unroll
        for (int c = 0; c < E; ++c) top = MaxOp::apply(top, fabsf(w[c]));
    }
    const RowScale r = row_scale(team_reduce<MaxOp, kTeam>(top, scratch), a.binary, kFiniteMax<T>);
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        float w[E];
        widen<T>(raw[v], w);
        store_byte_slab<E, kTeam>(q + row * a.q_stride, v * kTeam * E, me.lane, cols, bytes_of<E>(w, r), v < kVecs - 1);
    }
    if (me.lane == 0) scale[row] = r.scale;
}

template <typename T, int kTeam, int kVecs>
__global__ __launch_bounds__(kTeamBlock<kTeam>) void restore(T *__restrict__ x, const int8_t *__restrict__ q, const float *__restrict__ scale,
                                                             QuantArgs a)
{
    constexpr int E = kVec<T>, kTeams = kTeamBlock<kTeam> / kTeam;
    const Team<kTeam> me;
    const int cols = (int)a.cols;
    const int64_t row = (a.first + blockIdx.x) * kTeams + me.id;
    if (row >= a.rows) return;
    uint64_t raw[kVecs];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) raw[v] = load_byte_slab<E, kTeam>(q + row * a.q_stride, v * kTeam * E, me.lane, cols, v < kVecs - 1);
    const float s = scale[row];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        settle_bytes<E, kTeam>(raw[v], v * kTeam * E, me.lane, cols, v < kVecs - 1);
        float w[E];
        from_bytes<E>(raw[v], w);
#pragma unroll
        for (int c = 0; c < E; ++c) w[c] *= s;
        store_slab<T, kTeam>(x + row * a.x_stride, v * kTeam * E, me.lane, cols, narrow<T>(w), v < kVecs - 1, a.stream);
    }
}

}  // namespace cams_ops
