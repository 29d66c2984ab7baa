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

// `stream`, uniform: the access is not to be kept in the caches (see streamed() on the host side).  The empty statements keep the two
// forms apart, which the compiler would merge into one without the hint.
template <typename T> __device__ __forceinline__ v4u load_vec(const T *p, bool stream = false)
{
    v4u v;
    if (stream) {
        asm volatile("");
        v = __builtin_nontemporal_load(reinterpret_cast<const v4u_any *>(p));
        asm volatile("");
    } else {
        v = *reinterpret_cast<const v4u_any *>(p);
    }
    return v;
}
template <typename T> __device__ __forceinline__ void store_vec(T *p, const v4u &v, bool stream = false)
{
    if (stream) {
        asm volatile("");
        __builtin_nontemporal_store(v, reinterpret_cast<v4u_any *>(p));
        asm volatile("");
    } else {
        *reinterpret_cast<v4u_any *>(p) = v;
    }
}

// Makes the compiler take what is widened from `v` before and after for different values: a row held in registers is widened anew
// by each pass over it, instead of being kept in its wide form too.
__device__ __forceinline__ void rewiden(v4u &v) { asm volatile("" : "+v"(v)); }

template <typename T> __device__ __forceinline__ uint32_t bits1(T x);
template <> __device__ __forceinline__ uint32_t bits1<float>(float x) { return __float_as_uint(x); }
template <> __device__ __forceinline__ uint32_t bits1<bf16_t>(bf16_t x) { return x.v; }
template <> __device__ __forceinline__ uint32_t bits1<f16_t>(f16_t x) { return x.v; }

// base + at elements for a base that is uniform over the wavefront: the offset stays a 32-bit number of bytes beside a scalar address.
template <typename T> __device__ __forceinline__ const T *offset32(const T *base, int at)
{
    return reinterpret_cast<const T *>(reinterpret_cast<const char *>(base) + (uint32_t)at * (uint32_t)sizeof(T));
}
template <typename T> __device__ __forceinline__ T *offset32(T *base, int at)
{
    return reinterpret_cast<T *>(reinterpret_cast<char *>(base) + (uint32_t)at * (uint32_t)sizeof(T));
}

// --- a row in slabs ----------------------------------------------------------------------------------------------------
//
// A row that a team of kTeam lanes takes lies in slabs of kTeam vectors, lane after lane; `first` is a slab's first element.  A slab inside
// the row is loaded without a look at the lanes.  Where the row ends inside a lane's vector, the row's last whole vector is loaded
// instead and moved into place later, by settle_slab: element by element it took eight loads, each waited for before the next.
// The row (from its very start, wherever `row` points into it) has at least a vector's elements.
// sure: the slab is known to lie inside (a constant where loops are unrolled: all but the last slab of a row that just fits).

// Elements [at, at + kVec) of a row of `len` in the lanes with at < need (need <= len), not in place yet; the other lanes' are zero.
template <typename T, int kTeam>
__device__ __forceinline__ v4u load_slab(const T *row, int first, int lane, int len, int need, bool sure = false, bool stream = false)
{
    constexpr int E = kVec<T>;
    const int at = first + lane * E;
    if (sure || first + kTeam * E <= need) return load_vec(offset32(row, at), stream);
    v4u raw = {0u, 0u, 0u, 0u};
    if (at < need) raw = load_vec(row + min(at, len - E));
    return raw;
}

// Puts the elements of load_slab into place; those from `keep` on (keep <= len) become `fill`.
template <typename T, int kTeam>
__device__ __forceinline__ void settle_slab(v4u &raw, int first, int lane, int len, int keep, uint32_t fill, bool sure = false)
{
    constexpr int E = kVec<T>;
    if (sure || first + kTeam * E <= keep) return;
    if (first + kTeam * E > len) {
        const int late = first + lane * E - (len - E);
        if (late > 0) {                             // the vector ended with the row: `late` elements further down
            if constexpr (sizeof(T) == 2) {
                if (late & 4) raw = v4u{raw[2], raw[3], 0u, 0u};
                if (late & 2) raw = v4u{raw[1], raw[2], raw[3], 0u};
                if (late & 1)
                    raw = v4u{(raw[0] >> 16) | (raw[1] << 16), (raw[1] >> 16) | (raw[2] << 16), (raw[2] >> 16) | (raw[3] << 16), raw[3] >> 16};
            } else {
                if (late & 2) raw = v4u{raw[2], raw[3], 0u, 0u};
                if (late & 1) raw = v4u{raw[1], raw[2], raw[3], 0u};
            }
        }
    }
    // one lane is cut, those behind it are all fill; its masks are the same for the whole team
    const int kept = max(keep - first, 0), cut = kept / E, rest = kept % E;
    if (lane >= cut) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t mask, both = fill;
            if constexpr (sizeof(T) == 4) {
                mask = rest > q ? 0xffffffffu : 0u;
            } else {
                mask = rest >= 2 * q + 2 ? 0xffffffffu : rest == 2 * q + 1 ? 0xffffu : 0u;
                both |= fill << 16;
            }
            if (lane > cut) mask = 0u;
            raw[q] = (raw[q] & mask) | (both & ~mask);
        }
    }
}

typedef uint32_t v2u_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u_any __attribute__((aligned(2)));

template <typename T, int kTeam>
__device__ __forceinline__ void store_slab(T *row, int first, int lane, int len, const v4u &raw, bool sure = false, bool stream = false)
{
    constexpr int E = kVec<T>;
    const int at = first + lane * E;
    T *p = offset32(row, at);
    if (sure || first + kTeam * E <= len || at + E <= len) {
        store_vec(p, raw, stream);
    } else if (at < len) {                          // a binary number of elements is left
        const int rest = len - at;
        if constexpr (sizeof(T) == 4) {
            if (rest & 2) *reinterpret_cast<v2u_any *>(p) = v2u_any{raw[0], raw[1]};
            if (rest & 1) *reinterpret_cast<u_any *>(p + (rest & 2)) = (rest & 2) ? raw[2] : raw[0];
        } else {
            if (rest & 4) *reinterpret_cast<v2u_any *>(p) = v2u_any{raw[0], raw[1]};
            if (rest & 2) *reinterpret_cast<u_any *>(p + (rest & 4)) = (rest & 4) ? raw[2] : raw[0];
            const uint32_t last = (rest & 4) ? ((rest & 2) ? raw[3] : raw[2]) : ((rest & 2) ? raw[1] : raw[0]);
            if (rest & 1) reinterpret_cast<uint16_t *>(p)[rest & 6] = (uint16_t)last;
        }
    }
}

// Parameters (fp32) of the same elements: kVec<T> floats, zero past the row.
template <typename T, int kTeam>
__device__ __forceinline__ void load_params(float (&x)[kVec<T>], const float *p, int first, int lane, int len, bool sure = false)
{
    constexpr int E = kVec<T>;
    const int at = first + lane * E;
#pragma unroll
    for (int u = 0; u < E; u += 4) {
        v4u raw = load_slab<float, 1>(p, at + u, 0, len, len, sure);
        settle_slab<float, 1>(raw, at + u, 0, len, len, 0u, sure);
        float four[4];
        widen<float>(raw, four);
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

struct SumOp { static __device__ __forceinline__ float apply(float a, float b) { return a + b; } };
// NaN wins (v_maximum3_f32): a row with a NaN does not look like one without.
struct MaxOp { static __device__ __forceinline__ float apply(float a, float b) { return __builtin_elementwise_maximum(a, b); } };

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

// kValues reductions at once.  scratch: kValues * kTeam / 64 floats of LDS where kTeam > 64; there the workgroup meets at one barrier, and
// must meet at another one before the same scratch is used again.
template <typename Op, int kTeam, int kValues>
__device__ __forceinline__ void team_reduce(float (&v)[kValues], float *scratch)
{
    if constexpr (kTeam <= kWave) {
#pragma unroll
        for (int u = 0; u < kValues; ++u) v[u] = lanes_reduce<Op, kTeam>(v[u]);
    } else {
        constexpr int kWaves = kTeam / kWave;
#pragma unroll
        for (int u = 0; u < kValues; ++u) {
            v[u] = lanes_reduce<Op, kWave>(v[u]);
            if ((threadIdx.x & (kWave - 1)) == 0) scratch[u * kWaves + threadIdx.x / kWave] = v[u];
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kValues; ++u) {
            v[u] = scratch[u * kWaves];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) v[u] = Op::apply(v[u], scratch[u * kWaves + w]);
        }
    }
}
template <typename Op, int kTeam>
__device__ __forceinline__ float team_reduce(float v, float *scratch)
{
    float one[1] = {v};
    team_reduce<Op, kTeam, 1>(one, scratch);
    return one[0];
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

// Numbers below this size leave room within fp32 for their distances: scores in units of log 2 among each other; from any fp32 number, since half
// a unit of the largest is 2^103.
constexpr float kPlainMax = 1e31f;

// A distance to the maximum, (x - top) unit, costs one instruction as fma(x, unit, -c) with c = top unit rounded to fp32.  Every such distance is
// off by the same top unit - c, at most 1/2 while |c| < 2^24: sums of 2^distance are multiplied by kept_back() afterwards.  Beyond that (logits
// masked with a large finite number, as far as some lanes see nothing else) it would leave fp32, and x - top is formed first.
constexpr float kPlainProduct = 16777216.f;
__device__ __forceinline__ bool plain_product(float c) { return fabsf(c) < kPlainProduct; }        // false for a NaN
__device__ __forceinline__ float kept_back(float top, float unit, float c) { return __builtin_amdgcn_exp2f(fmaf(-top, unit, c)); }

// log sum exp((z - top) / T) of a row, or NaN where the row has no distribution: nothing but -infinity, or a +infinity.  Log probabilities are
// (z - top) / T - log_sum: lse = top / T + log_sum has lost what the size of top has no bits for.
__device__ __forceinline__ float log_sum(float top, float sum) { return fabsf(top) == INFINITY ? NAN : logf(sum); }
__device__ __forceinline__ float lse_value(const Lse &v, float inv_t) { return fmaf(v.top, inv_t, log_sum(v.top, v.sum)); }

}  // namespace cams_ops
