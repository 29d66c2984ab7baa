// Weight gradients of a linear layer from its input as it was kept in 8 bits, per worker.
//
//   dW[w][o][i] = sum over worker w's rows r of dy[r][o] (q[r][i] scale[r])
//
// The matrix instruction takes bfloat16, which holds q exactly (7 bits); what it cannot hold goes in several planes whose products are added up:
//   dy in bfloat16, scales powers of two     q scale and dy, both exact: one plane
//   dy in float16, scales powers of two      dy scale in two planes: its 11 bits are 8 and 3, so nothing is lost.  (The matrix instruction of half precision
//                                            would take both as they are, but it lines products up as if factors below 2^-14 were 2^-14 and cuts
//                                            them 24 bits below the largest: gradients of 2^-24 were off by 5e-5.)
//   dy in bfloat16, any scale                fl32(q scale) or fl32(dy scale), whichever makes less to write, in planes of 8 bits: three, all 24 bits, for
//                                            gradients in fp32; for gradients in 16 bits, whose own rounding is 2^-9 or 2^-12, two: 2^-17 of
//                                            each product is lost
//   dy in float16, any scale                 fl32(dy scale), the same
//   dy in float32                            fl32(dy scale) in three planes
// A first kernel writes q and the planes of dy as rows of bfloat16 (dy itself is read where one plane does and its rows are aligned), so that
// each number is widened once and not once for every tile that it meets.  The sum runs over planes and rows.  Both operands lie across it (their rows are the sum's
// index): a step's rows go from memory to LDS as they lie, without registers, and the transposing LDS reads hand every lane its column's
// values.
//
// 16384 rows, 4096 x 4096, four workers, bfloat16: 439 us with the first kernel, which takes 33 of them (HBM-bound, 6.1 TB/s); 1350 TFLOP/s for the
// product alone, bound by power as product8 is.  Widened tile by tile on the way to LDS the whole took 1159 us.  Half precision,
// 16000 rows, one worker, in two planes: 833 us (13698 rows, 192 x 3914, two workers: 148, most of it the planes' bytes).  bfloat16 with any scales, 6168
// rows, 183 x 4697, four workers, gradients in 16 bits: 80 us with two planes on q's side, 90 on dy's.  16384 rows, 768 x 2304, eight workers: 66 us, 216
// tiles for 256 compute units.
#pragma once
#include "product8_kernels.h"

namespace cams_ops {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

// x = hi + rest with 8 bits in hi.  Of an infinity nothing is left.
__device__ __forceinline__ float take_plane(float &x)
{
    const float hi = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    x = fabsf(x) == INFINITY ? 0.f : x - hi;
    return hi;
}

constexpr int kPrepareThreads = 256;

struct PrepareArgs {
    int64_t rows, cols, outs, q_stride, dy_stride;
    int64_t a_ld, b_ld, a_plane, b_plane;            // rows of the results, elements apart, and planes of them
    int64_t worker_rows, bias_rows;                  // rows of a worker, and of one of its pieces for the bias
    int lanes_a, lanes_b;                            // lanes that share a row, powers of two up to 256
    unsigned blocks_a, blocks_b;                     // workgroups for q and for dy; the others are for the bias
    unsigned bias_chunks;
    unsigned first;
};

// Numbers [c, c + 8) of a row of `cols`, zero behind it.  No branch goes round a load, so that those of several rows are on their way together:
// where the row ends inside, its last whole vectors are loaded and moved into place.
template <typename T>
__device__ __forceinline__ void load_eight(float (&x)[8], const T *row, int c, int cols)
{
    constexpr int E = kVec<T>;
    if (cols < E) {
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = c + u < cols ? widen1(row[c + u]) : 0.f;
        return;
    }
#pragma unroll
    for (int u = 0; u < 8; u += E) {
        v4u raw = load_vec(row + min(c + u, cols - E));
        settle_slab<T, 1>(raw, c + u, 0, cols, cols, 0u);
        float part[E];
        widen<T>(raw, part);
#pragma unroll
        for (int v = 0; v < E; ++v) x[u + v] = part[v];
    }
}

constexpr int kBiasParts = kPrepareThreads * 8 / kBiasCols;         // threads that share eight columns

// Sums of 256 columns of dy over a piece of a worker's rows, into sums[worker][piece][outs]: eight threads take every eighth row for the same
// eight columns, and their sums are added in order.
template <typename T>
__device__ __forceinline__ void bias_sums(float *__restrict__ sums, const T *__restrict__ dy, unsigned block, const PrepareArgs &a)
{
    __shared__ float parts[kBiasParts][kBiasCols];
    const unsigned blocks = (unsigned)((a.outs + kBiasCols - 1) / kBiasCols);
    const unsigned piece = block / blocks % a.bias_chunks, worker = block / blocks / a.bias_chunks;
    const int part = threadIdx.x / (kBiasCols / 8), lane = threadIdx.x % (kBiasCols / 8);
    const int64_t base = (int64_t)(block % blocks) * kBiasCols, c = base + lane * 8;
    const int64_t lo = piece * a.bias_rows, hi = min(lo + a.bias_rows, a.worker_rows);
    float s[8] = {};
    const T *from = dy + (worker * a.worker_rows + lo + part) * a.dy_stride;
    if (c < a.outs) {
#pragma unroll 4
        for (int64_t r = lo + part; r < hi; r += kBiasParts, from += kBiasParts * a.dy_stride) {
            float x[8];
            load_eight(x, from, (int)c, (int)a.outs);
#pragma unroll
            for (int u = 0; u < 8; ++u) s[u] += x[u];
        }
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) parts[part][lane * 8 + u] = s[u];
    __syncthreads();
    const int64_t col = base + threadIdx.x;
    if (col >= a.outs) return;
    float all = parts[0][threadIdx.x];
#pragma unroll
    for (int q = 1; q < kBiasParts; ++q) all += parts[q][threadIdx.x];
    sums[((int64_t)worker * a.bias_chunks + piece) * a.outs + col] = all;
}

// The pieces' sums of `threads` columns of a worker joined in order.
template <typename G>
__device__ __forceinline__ void bias_join(G *__restrict__ dbias, const float *__restrict__ sums, int64_t outs, unsigned pieces, int64_t grad_stride,
                                          int64_t worker, int64_t col)
{
    if (col >= outs) return;
    float sum = 0.f;
#pragma unroll 8
    for (unsigned q = 0; q < pieces; ++q) sum += sums[(worker * pieces + q) * outs + col];
    dbias[worker * grad_stride + col] = narrow1<G>(sum);
}

// Rows in 16 bits whose length is a multiple of eight (zeros behind the row): kQ planes of q scale where dy stays as it is (kD = 1), q otherwise; kD
// planes of dy scale, or dy itself.  kBias: further workgroups sum dy's columns.  Lanes that share a row take kPrepareRows rows, whose loads are on their way together: one after the other 16384 rows of 768 took 8.2 us in place of 7.4.
constexpr int kPrepareRows = 4;
template <typename T, int kQ, int kD, bool kBias>
__global__ __launch_bounds__(kPrepareThreads) void weight_prepare(bf16_t *__restrict__ a_out, bf16_t *__restrict__ b_out, float *__restrict__ sums,
                                                                  const T *__restrict__ dy, const int8_t *__restrict__ q,
                                                                  const float *__restrict__ scale, PrepareArgs a)
{
    unsigned block = a.first + blockIdx.x;
    if constexpr (kBias) {
        if (block >= a.blocks_a + a.blocks_b) {
            bias_sums<T>(sums, dy, block - a.blocks_a - a.blocks_b, a);
            return;
        }
    }
    const bool of_q = block < a.blocks_a;
    if (!of_q) block -= a.blocks_a;
    const int lanes = of_q ? a.lanes_a : a.lanes_b, beside = kPrepareThreads / lanes;     // rows that a workgroup takes at a time
    const int64_t row0 = (int64_t)block * beside * kPrepareRows + threadIdx.x / lanes;
    const int lane = threadIdx.x % lanes;
    int64_t row[kPrepareRows];
    float s[kPrepareRows];
#pragma unroll
    for (int u = 0; u < kPrepareRows; ++u) {
        row[u] = min(row0 + u * beside, a.rows - 1);             // rows behind the last one are the last one again
        s[u] = scale[row[u]];
    }
    if (of_q) {
        for (int64_t c = lane * 8; c < a.cols; c += lanes * 8) {
            uint64_t raw[kPrepareRows];
            if (a.cols >= 8) {
#pragma unroll
                for (int u = 0; u < kPrepareRows; ++u) raw[u] = load_bytes<8>(q + row[u] * a.q_stride + min(c, a.cols - 8));
#pragma unroll
                for (int u = 0; u < kPrepareRows; ++u) settle_bytes<8, 1>(raw[u], (int)c, 0, (int)a.cols, false);
            } else {
#pragma unroll
                for (int u = 0; u < kPrepareRows; ++u) {
                    raw[u] = 0;
                    for (int v = 0; c + v < a.cols; ++v) raw[u] |= (uint64_t)(uint8_t)q[row[u] * a.q_stride + c + v] << (8 * v);
                }
            }
#pragma unroll
            for (int u = 0; u < kPrepareRows; ++u) {
                float x[8];
                from_bytes<8>(raw[u], x);
                if constexpr (kD == 1) {
#pragma unroll
                    for (int v = 0; v < 8; ++v) x[v] *= s[u];
                }
#pragma unroll
                for (int p = 0; p < kQ; ++p) {
                    float plane[8];
#pragma unroll
                    for (int v = 0; v < 8; ++v) {
                        plane[v] = x[v];
                        if (p < kQ - 1) {
                            plane[v] = take_plane(x[v]);
                            if (x[v] == 0.f) x[v] = plane[v] * 0x1p-40f;         // an infinite dy meets no zero that was none
                        }
                    }
                    *reinterpret_cast<v4u *>(a_out + p * a.a_plane + row[u] * a.a_ld + c) = narrow<bf16_t>(plane);
                }
            }
        }
        return;
    }
    for (int64_t c = lane * 8; c < a.outs; c += lanes * 8) {
        float x[kPrepareRows][8];
#pragma unroll
        for (int u = 0; u < kPrepareRows; ++u) load_eight(x[u], dy + row[u] * a.dy_stride, (int)c, (int)a.outs);
#pragma unroll
        for (int u = 0; u < kPrepareRows; ++u) {
            if constexpr (kD > 1) {
#pragma unroll
                for (int v = 0; v < 8; ++v) x[u][v] *= s[u];
            }
#pragma unroll
            for (int p = 0; p < kD; ++p) {
                float plane[8];
#pragma unroll
                for (int v = 0; v < 8; ++v) plane[v] = p < kD - 1 ? take_plane(x[u][v]) : x[u][v];
                *reinterpret_cast<v4u *>(b_out + p * a.b_plane + row[u] * a.b_ld + c) = narrow<bf16_t>(plane);
            }
        }
    }
}

struct WeightArgs {
    int64_t cols, outs, a_ld, b_ld, a_plane, b_plane;
    int64_t worker_rows;
    int64_t out_stride, worker_stride, piece_stride; // of the result, in elements: its rows', the workers', the pieces'
    int tiles_i, tiles_o, n, planes;
    int splits, split_steps;                         // pieces of the sum over planes and steps of rows, and their length
    unsigned first;
    bool stream_out;                                 // the result is stored as a stream
    unsigned tiles;                                  // workgroups for tiles; the others join the bias' sums
    unsigned bias_chunks;
    int64_t grad_stride;
};

// A tile of kI input channels x kO output channels by kWavesI x kWavesO wavefronts.  kInFirst: the result is [i][o], otherwise [o][i].
//
// A transposing read takes 32 bytes, the 16 columns of a fragment, from rows 0..3 and 8..11 at a time, then from 16..19 and 24..27, and these are to lie in
// different banks: a row's 32-byte blocks stand at place block ^ (row & 3); where a load's 1024 bytes are two rows only, at block ^ (row & 1), and
// loads stand 64 bytes further apart; every eight rows another 128.  All fragments of a lane then lie at a few addresses and constant
// distances from them.  Stages as in product8.
template <typename G, bool kInFirst, int kI, int kO, int kWavesI, int kWavesO>
__global__ __launch_bounds__(kWavesI *kWavesO *kWave, 2) void weight_grad(G *__restrict__ out, G *__restrict__ dbias,
                                                                          const bf16_t *__restrict__ a_rows, const bf16_t *__restrict__ b_rows,
                                                                          const float *__restrict__ bias_sums, WeightArgs a)
{
    if (a.first + blockIdx.x >= a.tiles) {
        constexpr int kThreads = kWavesI * kWavesO * kWave;
        const unsigned id = a.first + blockIdx.x - a.tiles, blocks = (unsigned)((a.outs + kThreads - 1) / kThreads);
        bias_join<G>(dbias, bias_sums, a.outs, a.bias_chunks, a.grad_stride, id / blocks, (int64_t)(id % blocks) * kThreads + threadIdx.x);
        return;
    }
    constexpr int kWaves = kWavesI * kWavesO;
    constexpr int kIi = kI / kWavesI / 16, kOi = kO / kWavesO / 16;
    constexpr int kBytesI = kI * 2, kBytesO = kO * 2;                        // of a row in LDS
    constexpr int kRowsI = 1024 / kBytesI, kRowsO = 1024 / kBytesO;          // rows of a wavefront-wide load
    constexpr int kLoadsI = kWeightStep / kRowsI / kWaves, kLoadsO = kWeightStep / kRowsO / kWaves;
    static_assert(kLoadsI * kRowsI * kWaves == kWeightStep && kLoadsO * kRowsO * kWaves == kWeightStep, "whole loads");
    constexpr int kSwapI = kRowsI == 2 ? 1 : 3, kSwapO = kRowsO == 2 ? 1 : 3;
    constexpr int kLoadI = kRowsI == 2 ? 1088 : 1024, kLoadO = kRowsO == 2 ? 1088 : 1024;      // bytes from load to load in LDS
    constexpr int kEight = 128;                                                                // and besides from eight rows to the next
    constexpr int kPartI = kWeightStep / kRowsI * kLoadI + kWeightStep / 8 * kEight, kPartO = kWeightStep / kRowsO * kLoadO + kWeightStep / 8 * kEight;
    constexpr int kStages = kI + kO <= 128 ? 8 : 4;
    __shared__ __attribute__((aligned(1024))) int8_t tile[kStages][kPartI + kPartO];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    int set, ti, to;
    grouped_tile(a.first + blockIdx.x, (unsigned)(a.n * a.splits), a.tiles_i, a.tiles_o, set, ti, to);
    const int worker = set / a.splits, piece = set % a.splits;
    const int64_t i0 = (int64_t)ti * kI, o0 = (int64_t)to * kO;
    const bf16_t *at = a_rows + worker * a.worker_rows * a.a_ld + i0, *bt = b_rows + worker * a.worker_rows * a.b_ld + o0;
    const int rows = (int)a.worker_rows, steps = (rows + kWeightStep - 1) / kWeightStep;
    const int begin = piece * a.split_steps, end = min(steps * a.planes, begin + a.split_steps);

    // a lane's part of each load: its row, and the 16 bytes that belong to its place there
    constexpr uint32_t kNowhere = 0x80000000u;       // past the end of any buffer: reads zeros
    uint32_t off_i[kLoadsI], off_o[kLoadsO];
    auto offset = [&](int first, int row_bytes, int swap, int64_t left, int64_t ld) {
        const int row = first + lane / (row_bytes / 16), place = lane % (row_bytes / 16);
        const int column = ((place >> 1) ^ (row & swap)) * 16 + (place & 1) * 8;
        return column < left ? (uint32_t)((row * ld + column) * 2) : kNowhere;
    };
#pragma unroll
    for (int j = 0; j < kLoadsI; ++j) off_i[j] = offset((j * kWaves + wave) * kRowsI, kBytesI, kSwapI, a.cols - i0, a.a_ld);
#pragma unroll
    for (int j = 0; j < kLoadsO; ++j) off_o[j] = offset((j * kWaves + wave) * kRowsO, kBytesO, kSwapO, a.outs - o0, a.b_ld);
    int step = begin % max(steps, 1), unsent = end - begin;
    const bf16_t *a_next = at + begin / max(steps, 1) * a.a_plane + (int64_t)step * kWeightStep * a.a_ld;
    const bf16_t *b_next = bt + begin / max(steps, 1) * a.b_plane + (int64_t)step * kWeightStep * a.b_ld;
    const int64_t a_back = (int64_t)steps * kWeightStep * a.a_ld - a.a_plane, b_back = (int64_t)steps * kWeightStep * a.b_ld - a.b_plane;
    auto send = [&](int stage) {                     // the next step's rows, memory to LDS, asynchronous; zeros after the last one
        // buffers that end with the worker's last row
        const int left = unsent > 0 ? min(rows - step * kWeightStep, kWeightStep) : 0;
        --unsent;
        const v4u asrc = raw_buffer(a_next, (uint32_t)left * (uint32_t)a.a_ld * 2u);
        const v4u bsrc = raw_buffer(b_next, (uint32_t)left * (uint32_t)a.b_ld * 2u);
#pragma unroll
        for (int j = 0; j < kLoadsI; ++j) to_lds(asrc, off_i[j], &tile[stage][(j * kWaves + wave) * kLoadI + (j * kWaves + wave) * kRowsI / 8 * kEight]);
#pragma unroll
        for (int j = 0; j < kLoadsO; ++j) to_lds(bsrc, off_o[j], &tile[stage][kPartI + (j * kWaves + wave) * kLoadO + (j * kWaves + wave) * kRowsO / 8 * kEight]);
        a_next += kWeightStep * a.a_ld;
        b_next += kWeightStep * a.b_ld;
        if (++step == steps) {                       // the next plane
            step = 0;
            a_next -= a_back;
            b_next -= b_back;
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
    // A lane's eight values of the sum's index are rows 8 g .. 8 g + 7 for its group g.
    const int trow = fgroup * 8 + frow / 4;
    constexpr int kAtI = kIi < kSwapI + 1 ? kIi : kSwapI + 1, kAtO = kOi < kSwapO + 1 ? kOi : kSwapO + 1;
    int at_i[kAtI], at_o[kAtO];                      // of the first fragments
#pragma unroll
    for (int i = 0; i < kAtI; ++i)
        at_i[i] = trow / kRowsI * kLoadI + fgroup * kEight + trow % kRowsI * kBytesI + ((wi * kIi + i) ^ (trow & kSwapI)) * 32 + frow % 4 * 8;
#pragma unroll
    for (int o = 0; o < kAtO; ++o)
        at_o[o] = kPartI + trow / kRowsO * kLoadO + fgroup * kEight + trow % kRowsO * kBytesO + ((wo * kOi + o) ^ (trow & kSwapO)) * 32 + frow % 4 * 8;
    auto fragment = [&](const int8_t *low, int four_rows) {
        typedef __attribute__((address_space(3))) v4s lds_v4s;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)low);
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(low + four_rows));
        return __builtin_bit_cast(v8bf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    constexpr int kFourI = 4 * kBytesI + (kLoadI - 1024) * 4 / kRowsI, kFourO = 4 * kBytesO + (kLoadO - 1024) * 4 / kRowsO;
    struct Frags {
        v8bf i[kIi], o[kOi];
    };
    auto read = [&](Frags &f, int stage) {
#pragma unroll
        for (int o = 0; o < kOi; ++o) f.o[o] = fragment(&tile[stage][at_o[o % kAtO] + o / kAtO * kAtO * 32], kFourO);
#pragma unroll
        for (int i = 0; i < kIi; ++i) f.i[i] = fragment(&tile[stage][at_i[i % kAtI] + i / kAtI * kAtI * 32], kFourI);
    };
    auto multiply = [&](const Frags &f) {
#pragma unroll
        for (int i = 0; i < kIi; ++i)
#pragma unroll
            for (int o = 0; o < kOi; ++o) {
                if constexpr (kInFirst) acc[i][o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.o[o], f.i[i], acc[i][o], 0, 0, 0);
                else acc[i][o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.i[i], f.o[o], acc[i][o], 0, 0, 0);
            }
    };
    constexpr int kReads = 2 * (kIi + kOi), kPer = kIi * kOi / kReads;
    auto mixed = [&]() {
#pragma unroll
        for (int u = 0; u < kReads; ++u) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);          // a read from LDS
            __builtin_amdgcn_sched_group_barrier(0x008, kPer, 0);       // matrix instructions
        }
        __builtin_amdgcn_sched_group_barrier(0x008, kIi * kOi - kPer * kReads, 0);
    };
    constexpr int kLoads = kLoadsI + kLoadsO;
    auto advance = [&](int u, const Frags &now, Frags &next) {          // a step, as in product8
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kStages - 3) * kLoads) : "memory");
        send((u + kStages - 1) % kStages);
        read(next, (u + 1) % kStages);
        multiply(now);
        mixed();
        __builtin_amdgcn_sched_barrier(0);
    };
    Frags even, odd;
#pragma unroll
    for (int u = 0; u < kStages - 1; ++u) send(u);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((kStages - 2) * kLoads) : "memory");
    read(even, 0);
    for (int c = begin; c < end; c += kStages) {
#pragma unroll
        for (int u = 0; u < kStages; u += 2) {
            if (kStages > 4 && c + u >= end) break;
            advance(u, even, odd);
            advance(u + 1, odd, even);
        }
    }
    // nothing is on its way to LDS or read from it any more, by any wavefront
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    G *ot = out + worker * a.worker_stride + piece * a.piece_stride;
    constexpr int kAcross = kInFirst ? kIi : kOi, kAlong = kInFirst ? kOi : kIi;     // fragments across the result's rows and along them
    const int64_t across = kInFirst ? a.cols : a.outs, along = kInFirst ? a.outs : a.cols;
    const int64_t row0 = kInFirst ? i0 + wi * kIi * 16 : o0 + wo * kOi * 16, col0 = kInFirst ? o0 + wo * kOi * 16 : i0 + wi * kIi * 16;
    G *mine = reinterpret_cast<G *>(&tile[0][0]) + wave * 16 * kSixteenLd<G, kAlong>;
    static_assert(kWaves * 16 * kSixteenLd<G, kAlong> * sizeof(G) <= sizeof tile, "room for the results");
#pragma unroll
    for (int x = 0; x < kAcross; ++x) {
        const int64_t row = row0 + x * 16;
        G values[kAlong][4];
#pragma unroll
        for (int y = 0; y < kAlong; ++y)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float sum = kInFirst ? acc[kInFirst ? x : 0][kInFirst ? y : 0][c] : acc[kInFirst ? 0 : y][kInFirst ? 0 : x][c];
                values[y][c] = narrow1<G>(sum);
            }
        store_sixteen<G, kAlong>(mine, values, ot + row * a.out_stride + col0, a.out_stride, across - row, along - col0, a.stream_out);
    }
}

constexpr int kWeightJoinThreads = 256;

// The pieces' sums work[piece][worker][cells] joined in order into the workers' rows, four cells a thread; further workgroups join the bias' sums.
template <typename G>
__global__ __launch_bounds__(kWeightJoinThreads) void weight_join(G *__restrict__ out, G *__restrict__ dbias, const float *__restrict__ work,
                                                                  const float *__restrict__ bias_sums, int64_t cells, int splits,
                                                                  int64_t piece_stride, WeightArgs a)
{
    const unsigned block = a.first + blockIdx.x;
    if (block >= a.tiles) {
        bias_join<G>(dbias, bias_sums, a.outs, a.bias_chunks, a.grad_stride, blockIdx.y, (int64_t)(block - a.tiles) * kWeightJoinThreads + threadIdx.x);
        return;
    }
    const int64_t c = ((int64_t)block * kWeightJoinThreads + threadIdx.x) * 4;
    if (c >= cells) return;
    const float *in = work + (int64_t)blockIdx.y * cells + c;
    G *p = out + (int64_t)blockIdx.y * a.grad_stride + c;
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
