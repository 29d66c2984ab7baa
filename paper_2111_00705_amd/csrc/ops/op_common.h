// Shared device helpers of the operators in this folder: 16-byte accesses of fp32, bfloat16 and half-precision rows at any
// alignment of the element, and reductions over teams of lanes in a fixed order.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cams_ops {

constexpr int kWave = 64;

struct bf16_t { uint16_t v; };
struct f16_t { uint16_t v; };

// Elements of one 16-byte access.
template <typename T> constexpr int kVec = 16 / (int)sizeof(T);

// gfx950 takes a 16-byte global access at any alignment: a copy between addresses that are one 16-bit element off ran at
// 5.2 - 5.5 TB/s against 5.5 aligned, so rows of odd strides need no path of their own.
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(2)));

typedef float v2f __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float widen1(float x) { return x; }
__device__ __forceinline__ float widen1(bf16_t x) { return __uint_as_float((uint32_t)x.v << 16); }
__device__ __forceinline__ float widen1(f16_t x) { return (float)__builtin_bit_cast(_Float16, x.v); }

// Rounding to nearest even, the only one: a result is rounded once, where it is stored.
template <typename T> __device__ __forceinline__ T narrow1(float x);
template <> __device__ __forceinline__ float narrow1<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16_t narrow1<bf16_t>(float x) { return {__builtin_bit_cast(uint16_t, (__bf16)x)}; }
template <> __device__ __forceinline__ f16_t narrow1<f16_t>(float x) { return {__builtin_bit_cast(uint16_t, (_Float16)x)}; }

template <typename T> __device__ __forceinline__ void widen(const v4u &raw, float (&x)[kVec<T>]);
template <> __device__ __forceinline__ void widen<float>(const v4u &raw, float (&x)[4])
{
#pragma unroll
    for (int q = 0; q < 4; ++q) x[q] = __uint_as_float(raw[q]);
}
template <> __device__ __forceinline__ void widen<bf16_t>(const v4u &raw, float (&x)[8])
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        x[2 * q] = __uint_as_float(raw[q] << 16);
        x[2 * q + 1] = __uint_as_float(raw[q] & 0xffff0000u);
    }
}
template <> __device__ __forceinline__ void widen<f16_t>(const v4u &raw, float (&x)[8])
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const v2h h = __builtin_bit_cast(v2h, (uint32_t)raw[q]);
        x[2 * q] = (float)h[0];
        x[2 * q + 1] = (float)h[1];
    }
}

template <typename T> __device__ __forceinline__ v4u narrow(const float (&x)[kVec<T>]);
template <> __device__ __forceinline__ v4u narrow<float>(const float (&x)[4])
{
    return v4u{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}
template <> __device__ __forceinline__ v4u narrow<bf16_t>(const float (&x)[8])
{
    v4u r;
#pragma unroll
    for (int q = 0; q < 4; ++q) r[q] = __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{x[2 * q], x[2 * q + 1]}), v2bf));
    return r;
}
template <> __device__ __forceinline__ v4u narrow<f16_t>(const float (&x)[8])
{
    v4u r;
#pragma unroll
    for (int q = 0; q < 4; ++q) r[q] = __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{x[2 * q], x[2 * q + 1]}), v2h));
    return r;
}

template <typename T> __device__ __forceinline__ v4u load_vec(const T *p) { return *reinterpret_cast<const v4u_any *>(p); }
template <typename T> __device__ __forceinline__ void store_vec(T *p, const v4u &v) { *reinterpret_cast<v4u_any *>(p) = v; }

// Makes the compiler take what is widened from `v` before and after for different values: a row held in registers is widened anew
// by each pass over it, instead of being kept in its wide form too.
__device__ __forceinline__ void rewiden(v4u &v) { asm volatile("" : "+v"(v)); }

template <typename T> __device__ __forceinline__ uint32_t bits1(T x);
template <> __device__ __forceinline__ uint32_t bits1<float>(float x) { return __float_as_uint(x); }
template <> __device__ __forceinline__ uint32_t bits1<bf16_t>(bf16_t x) { return x.v; }
template <> __device__ __forceinline__ uint32_t bits1<f16_t>(f16_t x) { return x.v; }

// Element q of a raw vector replaced by `b` (q known at compile time).
template <typename T> __device__ __forceinline__ void put_bits(v4u &raw, int q, uint32_t b)
{
    if constexpr (sizeof(T) == 4) raw[q] = b;
    else raw[q >> 1] = (q & 1) ? ((raw[q >> 1] & 0xffffu) | (b << 16)) : ((raw[q >> 1] & 0xffff0000u) | b);
}

// Row elements [at, at + kVec) of a row of `len`, those outside [0, len) as `fill` bits.  Touches nothing outside the row.
template <typename T, typename I>      // I: int or int64_t
__device__ __forceinline__ v4u load_row(const T *row, I at, I len, uint32_t fill = 0u)
{
    constexpr int E = kVec<T>;
    if (at >= 0 && at + E <= len) return load_vec(row + at);
    const uint32_t both = sizeof(T) == 4 ? fill : (fill | (fill << 16));
    v4u raw = {both, both, both, both};
    if (at > -E && at < len) {
#pragma unroll
        for (int q = 0; q < E; ++q)
            if (at + q >= 0 && at + q < len) put_bits<T>(raw, q, bits1(row[at + q]));
    }
    return raw;
}
template <typename T, typename I>
__device__ __forceinline__ void store_row(T *row, I at, I len, const v4u &raw)
{
    constexpr int E = kVec<T>;
    if (at >= 0 && at + E <= len) {
        store_vec(row + at, raw);
        return;
    }
    if (at <= -E || at >= len) return;
#pragma unroll
    for (int q = 0; q < E; ++q)
        if (at + q >= 0 && at + q < len) {
            if constexpr (sizeof(T) == 4) row[at + q] = __uint_as_float(raw[q]);
            else row[at + q].v = (uint16_t)((q & 1) ? raw[q >> 1] >> 16 : raw[q >> 1]);
        }
}

// A row that a team of kTeam lanes holds in registers lies in slabs of kTeam vectors, lane after lane.  `first` is a slab's first
// element; a slab that lies inside [0, len) is loaded without a look at the lanes.  Offsets stay 32-bit beside the row's address.
template <typename T, int kTeam>
__device__ __forceinline__ v4u load_slab(const T *row, int first, int lane, int len, uint32_t fill = 0u)
{
    constexpr int E = kVec<T>;
    const int at = first + lane * E;
    if (first + kTeam * E <= len) return load_vec(reinterpret_cast<const T *>(reinterpret_cast<const char *>(row) + (uint32_t)at * (uint32_t)sizeof(T)));
    return load_row(row, at, len, fill);
}
template <typename T, int kTeam>
__device__ __forceinline__ void store_slab(T *row, int first, int lane, int len, const v4u &raw)
{
    constexpr int E = kVec<T>;
    const int at = first + lane * E;
    if (first + kTeam * E <= len) store_vec(reinterpret_cast<T *>(reinterpret_cast<char *>(row) + (uint32_t)at * (uint32_t)sizeof(T)), raw);
    else store_row(row, at, len, raw);
}
// Parameters (fp32) of the same elements: kVec<T> floats.
template <typename T, int kTeam>
__device__ __forceinline__ void load_params(float (&x)[kVec<T>], const float *p, int first, int lane, int len)
{
    constexpr int E = kVec<T>;
    const int at = first + lane * E;
#pragma unroll
    for (int u = 0; u < E; u += 4) {
        float four[4];
        widen<float>(load_row(p, at + u, len), four);
#pragma unroll
        for (int q = 0; q < 4; ++q) x[u + q] = four[q];
    }
}

// Which team of the workgroup a lane belongs to, and its place in the team.
template <int kTeam> struct Team {
    int id, lane;
    __device__ __forceinline__ Team()
    {
        if constexpr (kTeam >= kWave) id = __builtin_amdgcn_readfirstlane(threadIdx.x / kTeam);   // uniform: rows get scalar addresses
        else id = threadIdx.x / kTeam;
        lane = threadIdx.x & (kTeam - 1);
    }
};
// Threads of the workgroup that such teams share.
template <int kTeam> constexpr int kTeamBlock = kTeam > 256 ? kTeam : 256;

// --- reductions over a team of kTeam lanes (a power of two; a wavefront or less: lanes side by side; more: the whole
// workgroup).  Fixed trees: the result depends on the lanes' values only, and every lane of the team receives it. ---------

// fmaxf ignores NaN, and is one instruction: for maxima whose row shows a NaN elsewhere.
struct LaxMaxOp { static __device__ __forceinline__ float apply(float a, float b) { return fmaxf(a, b); } };
struct SumOp { static __device__ __forceinline__ float apply(float a, float b) { return a + b; } };
// NaN wins: a row with a NaN must not look like one without.
struct MaxOp { static __device__ __forceinline__ float apply(float a, float b) { return (a > b || a != a) ? a : b; } };

// The permutes that ride in a vector instruction: a neighbour, the other pair, the other four, the other eight of a row of sixteen
// lanes; then the four rows through scalar registers.  (Six __shfl_xor are six round trips through the LDS unit.)  Every lane of the
// rows that take part must be active.
template <int kCtrl> __device__ __forceinline__ float dpp(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), kCtrl, 0xf, 0xf, false));
}
__device__ __forceinline__ float lane_value(float v, int lane)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane));
}
template <typename Op, int kLanes>
__device__ __forceinline__ float lanes_reduce(float v)
{
    static_assert(kLanes == 16 || kLanes == 64, "a row of lanes or a wavefront");
    v = Op::apply(v, dpp<0xb1>(v));        // quad_perm [1,0,3,2]
    v = Op::apply(v, dpp<0x4e>(v));        // quad_perm [2,3,0,1]
    v = Op::apply(v, dpp<0x141>(v));       // row_half_mirror
    v = Op::apply(v, dpp<0x140>(v));       // row_mirror
    if constexpr (kLanes == 64)
        v = Op::apply(Op::apply(lane_value(v, 0), lane_value(v, 16)), Op::apply(lane_value(v, 32), lane_value(v, 48)));
    return v;
}

// scratch: kTeam / 64 floats of LDS where kTeam > 64, not touched again before the next barrier of the team's workgroup.
template <typename Op, int kTeam>
__device__ __forceinline__ float team_reduce(float v, float *scratch)
{
    if constexpr (kTeam <= kWave) {
        return lanes_reduce<Op, kTeam>(v);
    } else {
        constexpr int kWaves = kTeam / kWave;
        v = lanes_reduce<Op, kWave>(v);
        __syncthreads();                                   // whoever read the scratch before has done so
        if ((threadIdx.x & (kWave - 1)) == 0) scratch[threadIdx.x / kWave] = v;
        __syncthreads();
        v = scratch[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v = Op::apply(v, scratch[w]);
        return v;
    }
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Running maximum of a row and the sum of exp((z - top) / T), unit = log2(e) / T.  The maximum stays in the row's own units and
// is subtracted first: scores masked with the type's lowest value would leave fp32 if they were scaled before.
struct Lse {
    float top, sum;
};

__device__ __forceinline__ Lse lse_join(const Lse &a, const Lse &b, float unit)
{
    const float top = MaxOp::apply(a.top, b.top);
    // equal tops first: -infinity beside -infinity is an empty sum, not a NaN
    const float fa = a.top == top ? 1.f : __builtin_amdgcn_exp2f((a.top - top) * unit);
    const float fb = b.top == top ? 1.f : __builtin_amdgcn_exp2f((b.top - top) * unit);
    return {top, a.sum * fa + b.sum * fb};
}

// log sum exp(z / T) of a row, or NaN where the row has no distribution: nothing but -infinity, or a +infinity.
__device__ __forceinline__ float lse_value(const Lse &v, float inv_t)
{
    return fabsf(v.top) == INFINITY ? NAN : fmaf(v.top, inv_t, logf(v.sum));
}

}  // namespace cams_ops
