// Weight gradients of a linear layer from its input as it was kept in 8 bits, per worker.
//
//   dW[w][o][i] = sum over worker w's rows r of dy[r][o] (q[r][i] scale[r])
//
// Both operands lie across the sum (their rows are the sum's index): a step's 32 rows go to LDS as they lie, and the transposing LDS reads
// hand every lane its column's values.  The matrix instruction takes bfloat16, which holds q exactly (7 bits); what it cannot hold goes in several
// planes whose products are added up:
//   dy in bfloat16, scales powers of two     q scale and dy, both exact: one product
//   dy in bfloat16, any scale; in float16    fl32(dy scale) in two planes of 8 bits: 2^-17 of each product is lost, nothing where the
//                                            scale is a power of two
//   dy in float32                            the same in three planes: all 24 bits
#pragma once
#include "product8_kernels.h"

namespace cams_ops {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));

struct WeightArgs {
    int64_t cols, outs, dy_stride, q_stride;
    int64_t worker_rows, split_rows;                 // rows of a worker, and of one of its pieces (a multiple of kWeightStep)
    int64_t out_stride, worker_stride, piece_stride; // of the result, in elements: its rows', the workers', the pieces'
    int tiles_i, tiles_o, n, splits;
    unsigned first;
};

constexpr int kWeightStep = 32, kWeightPad = 16;

template <typename T, bool kBinary> constexpr int kPlanes = sizeof(T) == 4 ? 3 : 2;
template <> constexpr int kPlanes<bf16_t, true> = 1;

// Eight values in bfloat16.
__device__ __forceinline__ v4u pack8(const float (&x)[8]) { return narrow<bf16_t>(x); }

// x = hi + rest with 8 bits in hi.  Of an infinity nothing is left.
__device__ __forceinline__ float take_plane(float &x)
{
    const float hi = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    x = fabsf(x) == INFINITY ? 0.f : x - hi;
    return hi;
}

// A tile of kI input channels x kO output channels by kWavesI x kWavesO wavefronts.  kInFirst: the result is [i][o], otherwise [o][i].
template <typename T, typename G, bool kBinary, bool kInFirst, int kI, int kO, int kWavesI, int kWavesO>
__global__ __launch_bounds__(kWavesI *kWavesO *kWave) void weight_grad(G *__restrict__ out, const T *__restrict__ dy, const int8_t *__restrict__ q,
                                                                       const float *__restrict__ scale, WeightArgs a)
{
    constexpr int kThreads = kWavesI * kWavesO * kWave, kP = kPlanes<T, kBinary>, E = kVec<T>;
    constexpr int kIi = kI / kWavesI / 16, kOi = kO / kWavesO / 16;
    constexpr int kLdI = kI + kWeightPad, kLdO = kO + kWeightPad;
    constexpr int kRowI = kI / 16, kRowO = kO / E;                           // 16-byte chunks of a row
    constexpr int kLoadsI = kWeightStep * kRowI / kThreads, kLoadsO = kWeightStep * kRowO / kThreads;
    static_assert(kLoadsI * kThreads == kWeightStep * kRowI && kLoadsO * kThreads == kWeightStep * kRowO, "whole loads");
    __shared__ __attribute__((aligned(16))) uint16_t q_lds[2][kWeightStep * kLdI];
    __shared__ __attribute__((aligned(16))) uint16_t dy_lds[2][kP][kWeightStep * kLdO];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    int set, ti, to;
    grouped_tile(a.first + blockIdx.x, (unsigned)(a.n * a.splits), a.tiles_i, a.tiles_o, set, ti, to);
    const int worker = set / a.splits, piece = set % a.splits;
    const int64_t i0 = (int64_t)ti * kI, o0 = (int64_t)to * kO;
    const int64_t r0 = (int64_t)piece * a.split_rows;
    const int rows = (int)min(a.split_rows, a.worker_rows - r0);
    const int64_t base = worker * a.worker_rows + r0;
    const int8_t *qt = q + base * a.q_stride;
    const T *dyt = dy + base * a.dy_stride;
    const float *st = scale + base;

    v4i qreg[kLoadsI], dyreg[kLoadsO];
    float qs[kLoadsI], dys[kLoadsO];
    auto load = [&](int r) {
#pragma unroll
        for (int j = 0; j < kLoadsI; ++j) {
            const int id = threadIdx.x + j * kThreads, row = r + id / kRowI;
            qreg[j] = v4i{0, 0, 0, 0};
            qs[j] = 0.f;
            if (row < rows) {
                qreg[j] = load_row16(qt + row * a.q_stride + i0, id % kRowI * 16, (int)min(a.cols - i0, (int64_t)kI));
                if constexpr (kP == 1) qs[j] = st[row];
            }
        }
#pragma unroll
        for (int j = 0; j < kLoadsO; ++j) {
            const int id = threadIdx.x + j * kThreads, row = r + id / kRowO;
            dyreg[j] = v4i{0, 0, 0, 0};
            dys[j] = 0.f;
            if (row < rows) {
                dyreg[j] = load_row16(reinterpret_cast<const int8_t *>(dyt + row * a.dy_stride + o0), id % kRowO * 16,
                                      (int)min(a.outs - o0, (int64_t)kO) * (int)sizeof(T));
                if constexpr (kP > 1) dys[j] = st[row];
            }
        }
    };
    auto put = [&](int stage) {
#pragma unroll
        for (int j = 0; j < kLoadsI; ++j) {
            const int id = threadIdx.x + j * kThreads;
            uint16_t *to_lds = &q_lds[stage][id / kRowI * kLdI + id % kRowI * 16];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float x[8];
                from_bytes<8>(((uint64_t)(uint32_t)qreg[j][2 * h + 1] << 32) | (uint32_t)qreg[j][2 * h], x);
                if constexpr (kP == 1) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) x[c] *= qs[j];
                }
                *reinterpret_cast<v4u *>(to_lds + 8 * h) = pack8(x);
            }
        }
#pragma unroll
        for (int j = 0; j < kLoadsO; ++j) {
            const int id = threadIdx.x + j * kThreads, at = id / kRowO * kLdO + id % kRowO * E;
            if constexpr (kP == 1) {
                *reinterpret_cast<v4i *>(&dy_lds[stage][0][at]) = dyreg[j];
            } else {
                float x[E], plane[8] = {};
                widen<T>(__builtin_bit_cast(v4u, dyreg[j]), x);
#pragma unroll
                for (int c = 0; c < E; ++c) x[c] *= dys[j];
#pragma unroll
                for (int p = 0; p < kP; ++p) {
#pragma unroll
                    for (int c = 0; c < E; ++c) plane[c] = p < kP - 1 ? take_plane(x[c]) : x[c];
                    const v4u bits = pack8(plane);
                    if constexpr (E == 8) *reinterpret_cast<v4u *>(&dy_lds[stage][p][at]) = bits;
                    else *reinterpret_cast<uint64_t *>(&dy_lds[stage][p][at]) = ((uint64_t)bits[1] << 32) | bits[0];
                }
            }
        }
    };

    v4f acc[kIi][kOi];
#pragma unroll
    for (int i = 0; i < kIi; ++i)
#pragma unroll
        for (int o = 0; o < kOi; ++o) acc[i][o] = v4f{0.f, 0.f, 0.f, 0.f};
    const int wi = wave / kWavesO, wo = wave % kWavesO;
    const int frow = lane & 15, fgroup = lane >> 4;
    // Transposing read: the 16 lanes of a group point at four rows of 16 columns, 8 bytes each; lane c of them receives column c of the four.
    const int trow = fgroup * 8 + frow / 4, tcol = frow % 4 * 4;
    auto fragment = [&](const uint16_t *p, int ld) {
        typedef __attribute__((address_space(3))) v4s *lds_v4s;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(uintptr_t)(__attribute__((address_space(3))) void *)(void *)p);
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(uintptr_t)(__attribute__((address_space(3))) void *)(void *)(p + 4 * ld));
        return __builtin_bit_cast(v8bf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto work_on = [&](int stage) {
        v8bf qf[kIi];
#pragma unroll
        for (int i = 0; i < kIi; ++i) qf[i] = fragment(&q_lds[stage][trow * kLdI + (wi * kIi + i) * 16 + tcol], kLdI);
#pragma unroll
        for (int p = kP - 1; p >= 0; --p)
#pragma unroll
            for (int o = 0; o < kOi; ++o) {
                const v8bf df = fragment(&dy_lds[stage][p][trow * kLdO + (wo * kOi + o) * 16 + tcol], kLdO);
#pragma unroll
                for (int i = 0; i < kIi; ++i) {
                    if constexpr (kInFirst) acc[i][o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(df, qf[i], acc[i][o], 0, 0, 0);
                    else acc[i][o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[i], df, acc[i][o], 0, 0, 0);
                }
            }
    };

    if (rows > 0) {
        load(0);
        put(0);
    }
    int stage = 0;
    for (int r = 0; r < rows; r += kWeightStep, stage ^= 1) {
        __syncthreads();
        const bool more = r + kWeightStep < rows;
        if (more) load(r + kWeightStep);
        work_on(stage);
        if (more) put(stage ^ 1);
    }

    G *ot = out + worker * a.worker_stride + piece * a.piece_stride;
    const int64_t across = kInFirst ? a.cols : a.outs, along = kInFirst ? a.outs : a.cols;
#pragma unroll
    for (int i = 0; i < kIi; ++i)
#pragma unroll
        for (int o = 0; o < kOi; ++o) {
            const int64_t ci = i0 + (wi * kIi + i) * 16, co = o0 + (wo * kOi + o) * 16;
            const int64_t row = (kInFirst ? ci : co) + frow, at = (kInFirst ? co : ci) + fgroup * 4;
            if (row >= across || at >= along) continue;
            G *p = ot + row * a.out_stride + at;
            G four[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) four[c] = narrow1<G>(acc[i][o][c]);
            if (at + 4 <= along) {
                if constexpr (sizeof(G) == 4) *reinterpret_cast<v4u_any *>(p) = v4u{bits1(four[0]), bits1(four[1]), bits1(four[2]), bits1(four[3])};
                else *reinterpret_cast<v2u_any *>(p) = v2u_any{bits1(four[0]) | (bits1(four[1]) << 16), bits1(four[2]) | (bits1(four[3]) << 16)};
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (at + c < along) p[c] = four[c];
            }
        }
}

constexpr int kWeightJoinThreads = 256;

// The pieces' sums work[piece][worker][cells] joined in order into the workers' rows, four cells a thread.
template <typename G>
__global__ __launch_bounds__(kWeightJoinThreads) void weight_join(G *__restrict__ out, const float *__restrict__ work, int64_t cells, int splits,
                                                                  int64_t piece_stride, int64_t worker_stride, unsigned first)
{
    const int64_t c = ((int64_t)(first + blockIdx.x) * kWeightJoinThreads + threadIdx.x) * 4;
    if (c >= cells) return;
    const float *in = work + (int64_t)blockIdx.y * cells + c;
    G *p = out + (int64_t)blockIdx.y * worker_stride + c;
    if (c + 4 <= cells) {
        v4f sum = {0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < splits; ++s) sum += __builtin_bit_cast(v4f, *reinterpret_cast<const v4u_any *>(in + s * piece_stride));
#pragma unroll
        for (int q = 0; q < 4; ++q) p[q] = narrow1<G>(sum[q]);
    } else {
        for (int q = 0; c + q < cells; ++q) {
            float sum = 0.f;
            for (int s = 0; s < splits; ++s) sum += in[s * piece_stride + q];
            p[q] = narrow1<G>(sum);
        }
    }
}

}  // namespace cams_ops
