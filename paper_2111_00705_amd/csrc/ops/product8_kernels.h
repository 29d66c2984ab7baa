// Product of 8-bit integers with a scale for each token and channel.
//
//   y[m][n] = (sum_k x[m][k] w[n][k]) x_scale[m] w_scale[n] + bias[n]
//
// The sums are 32-bit integers and exact in any order (fewer than 2^17 products of at most 2^14).
// Both operands lie along k, so a tile's rows go to LDS as they are, 128 bytes a row in eight 16-byte chunks; chunk c of row r stands at
// place c ^ (r & 7), which spreads the 16 rows of a fragment over all banks.  The matrix instruction takes the channels as its rows: a lane then
// holds four neighbouring channels of one token, which leave in one store.
#pragma once
#include "rows8.h"

namespace cams_ops {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) int8_t lds_bytes;

struct ProductArgs {
    int64_t rows, outs, x_stride, w_stride, y_stride;
    int cols;                    // k
    int tiles_m, tiles_n;
    int splits, k_split;         // pieces of k and their length, a multiple of kProductStep
    unsigned first;
};

constexpr int kProductStep = 128;        // bytes of k that a tile's rows hold in LDS
constexpr int kXcds = 8;

// 16 bytes of a row of `cols`, from k on; zero past the row.  Any alignment.
__device__ __forceinline__ v4i load_row16(const int8_t *row, int k, int cols)
{
    if (k + 16 <= cols) return __builtin_bit_cast(v4i, *reinterpret_cast<const v4u_1 *>(row + k));
    v4i v = {0, 0, 0, 0};
    if (k >= cols) return v;
    if (cols >= 16) {                                // the row's last 16 bytes, moved down
        const v4u t = *reinterpret_cast<const v4u_1 *>(row + cols - 16);
        const int late = k + 16 - cols;
        uint64_t lo = ((uint64_t)t[1] << 32) | t[0], hi = ((uint64_t)t[3] << 32) | t[2];
        if (late >= 8) {
            lo = hi >> (8 * (late - 8));
            hi = 0;
        } else {
            lo = (lo >> (8 * late)) | (hi << (64 - 8 * late));
            hi >>= 8 * late;
        }
        v = v4i{(int)(uint32_t)lo, (int)(uint32_t)(lo >> 32), (int)(uint32_t)hi, (int)(uint32_t)(hi >> 32)};
    } else {
        for (int q = 0; k + q < cols; ++q) {
            const int b = (int)(uint32_t)(uint8_t)row[k + q] << (8 * (q & 3));
            if (q < 4) v[0] |= b;
            else if (q < 8) v[1] |= b;
            else if (q < 12) v[2] |= b;
            else v[3] |= b;
        }
    }
    return v;
}

// Four neighbouring channels from n on of token m.
template <typename Y>
__device__ __forceinline__ void store_channels(Y *y, const v4i &acc, float xs, const float (&ws)[4], const float (&b)[4], int64_t m, int64_t n,
                                               const ProductArgs &a)
{
    Y out[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) out[q] = narrow1<Y>((float)acc[q] * xs * ws[q] + b[q]);
    Y *p = y + m * a.y_stride + n;
    if (n + 4 <= a.outs) {
        if constexpr (sizeof(Y) == 4) {
            *reinterpret_cast<v4u_any *>(p) = v4u{bits1(out[0]), bits1(out[1]), bits1(out[2]), bits1(out[3])};
        } else {
            *reinterpret_cast<v2u_any *>(p) = v2u_any{bits1(out[0]) | (bits1(out[1]) << 16), bits1(out[2]) | (bits1(out[3]) << 16)};
        }
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (n + q < a.outs) p[q] = out[q];
    }
}

__device__ __forceinline__ void load_channels(float (&v)[4], const float *p, int64_t n, int64_t outs)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = p && n + q < outs ? p[n + q] : 0.f;
}

// Which tile a workgroup takes, of `sets` sets of tiles_m x tiles_n: workgroups go round the XCDs, so each XCD gets a contiguous run of tiles,
// and a run goes through groups of eight tile rows, tile column by tile column, so that what its L2 holds of both operands is used again.
__device__ __forceinline__ void grouped_tile(unsigned block, unsigned sets, int tiles_m, int tiles_n, int &set, int &tm, int &tn)
{
    const unsigned tiles = (unsigned)tiles_m * (unsigned)tiles_n, all = tiles * sets;
    const unsigned per = all / kXcds, rest = all % kXcds, xcd = block % kXcds;
    const unsigned whole = xcd * per + min(xcd, rest) + block / kXcds;
    const unsigned id = whole % tiles;
    constexpr unsigned kGroup = 8;
    const unsigned group = id / (kGroup * tiles_n), within = id % (kGroup * tiles_n);
    const unsigned high = min(kGroup, (unsigned)tiles_m - group * kGroup);
    set = (int)(whole / tiles);
    tm = (int)(group * kGroup + within % high);
    tn = (int)(within / high);
}

// A tile of kM tokens x kN channels by kWavesM x kWavesN wavefronts.  kAsync: rows, strides and sizes are multiples of 16 bytes, and the tiles
// go from memory to LDS without registers; otherwise through registers, by loads of any alignment.
// kSplit: a piece of k; the sums go to work[piece][rows][outs].
template <typename Y, int kM, int kN, int kWavesM, int kWavesN, bool kAsync, bool kSplit>
__global__ __launch_bounds__(kWavesM *kWavesN *kWave) void product8(Y *__restrict__ y, int *__restrict__ work, const int8_t *__restrict__ x,
                                                                    const float *__restrict__ x_scale, const int8_t *__restrict__ w,
                                                                    const float *__restrict__ w_scale, const float *__restrict__ bias,
                                                                    ProductArgs a)
{
    constexpr int kWaves = kWavesM * kWavesN, kRows = kM + kN;
    constexpr int kMi = kM / kWavesM / 16, kNi = kN / kWavesN / 16;
    constexpr int kLoads = kRows / 8 / kWaves, kLoadsX = kM / 8 / kWaves;     // wavefront-wide loads of eight rows each
    static_assert(kM % (8 * kWaves) == 0 && kN % (8 * kWaves) == 0, "whole loads");
    __shared__ __attribute__((aligned(16))) int8_t tile[2][kRows * kProductStep];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const unsigned block = a.first + blockIdx.x;
    int piece, tm, tn;
    grouped_tile(block, (unsigned)a.splits, a.tiles_m, a.tiles_n, piece, tm, tn);
    const int64_t m0 = (int64_t)tm * kM, n0 = (int64_t)tn * kN;
    const int rows_m = (int)min((int64_t)kM, a.rows - m0), rows_n = (int)min((int64_t)kN, a.outs - n0);
    const int k_begin = kSplit ? piece * a.k_split : 0, k_end = kSplit ? min(a.cols, k_begin + a.k_split) : a.cols;
    const int8_t *xt = x + m0 * a.x_stride, *wt = w + n0 * a.w_stride;

    // lane's part of a load: row lane / 8 of the eight, the chunk that belongs to place lane % 8
    const int sub = lane >> 3, chunk = (lane & 7) ^ sub;
    constexpr uint32_t kNowhere = 0x80000000u;       // past the end of any tile: reads zeros
    uint32_t off[kLoads];
    // raw buffers of 32-bit data that end with the tile's last row
    const __amdgpu_buffer_rsrc_t xsrc =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(xt), 0, (uint32_t)((rows_m - 1) * a.x_stride + a.cols), 0x00020000);
    const __amdgpu_buffer_rsrc_t wsrc =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(wt), 0, (uint32_t)((rows_n - 1) * a.w_stride + a.cols), 0x00020000);
    v4i regs[kAsync ? 1 : kLoads];
    if constexpr (kAsync) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const bool of_x = j < kLoadsX;
            const int row = ((of_x ? j : j - kLoadsX) * kWaves + wave) * 8 + sub;
            off[j] = row < (of_x ? rows_m : rows_n) ? (uint32_t)(row * (of_x ? a.x_stride : a.w_stride) + chunk * 16) : kNowhere;
        }
    }
    auto place = [&](int j) {                        // first byte in LDS of load j
        return ((j < kLoadsX ? j * kWaves : kM / 8 + (j - kLoadsX) * kWaves) + wave) * 8 * kProductStep;
    };
    auto send = [&](int stage, int k) {              // memory to LDS, asynchronous
        const bool whole = k + kProductStep <= k_end;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            uint32_t at = off[j] + (uint32_t)k;
            if (!whole && k + chunk * 16 >= k_end) at = kNowhere;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(j < kLoadsX ? xsrc : wsrc, (lds_bytes *)&tile[stage][place(j)], 16, at, 0, 0, 0);
        }
    };
    auto load = [&](int k) {                         // memory to registers
        if constexpr (!kAsync) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const bool of_x = j < kLoadsX;
                const int row = ((of_x ? j : j - kLoadsX) * kWaves + wave) * 8 + sub;
                regs[j] = v4i{0, 0, 0, 0};
                if (row < (of_x ? rows_m : rows_n))
                    regs[j] = load_row16(of_x ? xt + row * a.x_stride : wt + row * a.w_stride, k + chunk * 16, k_end);
            }
        }
    };
    auto put = [&](int stage) {                      // registers to LDS
        if constexpr (!kAsync) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) *reinterpret_cast<v4i *>(&tile[stage][place(j) + lane * 16]) = regs[j];
        }
    };

    v4i acc[kNi][kMi];
#pragma unroll
    for (int n = 0; n < kNi; ++n)
#pragma unroll
        for (int m = 0; m < kMi; ++m) acc[n][m] = v4i{0, 0, 0, 0};
    const int wm = wave / kWavesN, wn = wave % kWavesN;
    const int frow = lane & 15, fgroup = lane >> 4, fswap = frow & 7;
    auto work_on = [&](int stage) {
        const int8_t *xs = &tile[stage][(wm * kMi * 16 + frow) * kProductStep];
        const int8_t *ws = &tile[stage][(kM + wn * kNi * 16 + frow) * kProductStep];
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const int at = ((kk * 4 + fgroup) ^ fswap) * 16;
            v4i wf[kNi], xf[kMi];
#pragma unroll
            for (int n = 0; n < kNi; ++n) wf[n] = *reinterpret_cast<const v4i *>(ws + n * 16 * kProductStep + at);
#pragma unroll
            for (int m = 0; m < kMi; ++m) xf[m] = *reinterpret_cast<const v4i *>(xs + m * 16 * kProductStep + at);
#pragma unroll
            for (int n = 0; n < kNi; ++n)
#pragma unroll
                for (int m = 0; m < kMi; ++m) acc[n][m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[n], xf[m], acc[n][m], 0, 0, 0);
        }
    };

    int stage = 0;
    if constexpr (kAsync) {
        send(0, k_begin);
        for (int k = k_begin; k < k_end; k += kProductStep, stage ^= 1) {
            // this stage has arrived, for every wavefront, and nobody reads the other one any more
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (k + kProductStep < k_end) send(stage ^ 1, k + kProductStep);
            work_on(stage);
        }
    } else {
        load(k_begin);
        put(0);
        for (int k = k_begin; k < k_end; k += kProductStep, stage ^= 1) {
            __syncthreads();
            const bool more = k + kProductStep < k_end;
            if (more) load(k + kProductStep);
            work_on(stage);
            if (more) put(stage ^ 1);
        }
    }

#pragma unroll
    for (int n = 0; n < kNi; ++n) {
        const int64_t at_n = n0 + (wn * kNi + n) * 16 + fgroup * 4;
        float ws[4], b[4];
        if constexpr (!kSplit) {
            load_channels(ws, w_scale, at_n, a.outs);
            load_channels(b, bias, at_n, a.outs);
        }
#pragma unroll
        for (int m = 0; m < kMi; ++m) {
            const int64_t at_m = m0 + (wm * kMi + m) * 16 + frow;
            if (at_m >= a.rows || at_n >= a.outs) continue;
            if constexpr (kSplit) {
                int *p = work + ((int64_t)piece * a.rows + at_m) * a.outs + at_n;
                if (at_n + 4 <= a.outs) {
                    *reinterpret_cast<v4u_any *>(p) = __builtin_bit_cast(v4u, acc[n][m]);
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (at_n + q < a.outs) p[q] = acc[n][m][q];
                }
            } else {
                store_channels<Y>(y, acc[n][m], x_scale[at_m], ws, b, at_m, at_n, a);
            }
        }
    }
}

constexpr int kProductThreads = 256;

// The pieces' sums joined, four channels a thread.
template <typename Y>
__global__ __launch_bounds__(kProductThreads) void product8_join(Y *__restrict__ y, const int *__restrict__ work, const float *__restrict__ x_scale,
                                                                 const float *__restrict__ w_scale, const float *__restrict__ bias, ProductArgs a)
{
    const int64_t quads = (a.outs + 3) / 4;
    const int64_t id = (int64_t)(a.first + blockIdx.x) * kProductThreads + threadIdx.x;
    if (id >= quads * a.rows) return;
    const int64_t m = id / quads, n = id % quads * 4;
    v4i sum = {0, 0, 0, 0};
    for (int s = 0; s < a.splits; ++s) {
        const int *p = work + ((int64_t)s * a.rows + m) * a.outs + n;
        if (n + 4 <= a.outs) {
            sum += __builtin_bit_cast(v4i, *reinterpret_cast<const v4u_any *>(p));
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (n + q < a.outs) sum[q] += p[q];
        }
    }
    float ws[4], b[4];
    load_channels(ws, w_scale, n, a.outs);
    load_channels(b, bias, n, a.outs);
    store_channels<Y>(y, sum, x_scale[m], ws, b, m, n, a);
}

// Few tokens: the weights' bytes count.  A workgroup takes 16 channels and all tokens (16 kMi at most), its wavefronts every kFewWaves-th step
// of k, and joins their sums in LDS.  Fragments come from memory as they are needed: a lane reads 32 bytes of a row in a step, so that four
// lanes use up a line; which k meet in an instruction does not matter as long as both operands agree.
constexpr int kFewWaves = 8, kFewStep = 128;
template <typename Y, int kMi>
__global__ __launch_bounds__(kFewWaves *kWave) void product8_few(Y *__restrict__ y, const int8_t *__restrict__ x, const float *__restrict__ x_scale,
                                                                 const int8_t *__restrict__ w, const float *__restrict__ w_scale,
                                                                 const float *__restrict__ bias, ProductArgs a)
{
    __shared__ v4i sums[kFewWaves][kMi][kWave];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int64_t n0 = (int64_t)(a.first + blockIdx.x) * 16;
    const int frow = lane & 15, fgroup = lane >> 4;
    const int8_t *wr = w + min(n0 + frow, a.outs - 1) * a.w_stride + fgroup * 32;
    const int8_t *xr[kMi];
#pragma unroll
    for (int m = 0; m < kMi; ++m) xr[m] = x + min((int64_t)m * 16 + frow, a.rows - 1) * a.x_stride + fgroup * 32;
    v4i acc[kMi];
#pragma unroll
    for (int m = 0; m < kMi; ++m) acc[m] = v4i{0, 0, 0, 0};
    const int whole = a.cols / kFewStep;
    constexpr int kAhead = kMi == 1 ? 4 : 2;         // steps whose loads are under way together
    int s = wave;
    for (; s + (kAhead - 1) * kFewWaves < whole; s += kAhead * kFewWaves) {
        v4i wf[kAhead][2], xf[kAhead][kMi][2];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = (s + u * kFewWaves) * kFewStep + h * 16;
                wf[u][h] = __builtin_bit_cast(v4i, *reinterpret_cast<const v4u_1 *>(wr + at));
#pragma unroll
                for (int m = 0; m < kMi; ++m) xf[u][m][h] = __builtin_bit_cast(v4i, *reinterpret_cast<const v4u_1 *>(xr[m] + at));
            }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int m = 0; m < kMi; ++m) acc[m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[u][h], xf[u][m][h], acc[m], 0, 0, 0);
    }
    for (; s * kFewStep < a.cols; s += kFewWaves) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = s * kFewStep + h * 16, left = a.cols - fgroup * 32;
            const v4i wf = load_row16(wr, at, left);
#pragma unroll
            for (int m = 0; m < kMi; ++m) acc[m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf, load_row16(xr[m], at, left), acc[m], 0, 0, 0);
        }
    }
#pragma unroll
    for (int m = 0; m < kMi; ++m) sums[wave][m][lane] = acc[m];
    __syncthreads();
    for (int id = threadIdx.x; id < kMi * kWave; id += kFewWaves * kWave) {
        const int m = id / kWave, l = id % kWave;
        v4i sum = sums[0][m][l];
#pragma unroll
        for (int v = 1; v < kFewWaves; ++v) sum += sums[v][m][l];
        const int64_t at_m = m * 16 + (l & 15), at_n = n0 + (l >> 4) * 4;
        if (at_m >= a.rows || at_n >= a.outs) continue;
        float ws[4], b[4];
        load_channels(ws, w_scale, at_n, a.outs);
        load_channels(b, bias, at_n, a.outs);
        store_channels<Y>(y, sum, x_scale[at_m], ws, b, at_m, at_n, a);
    }
}

}  // namespace cams_ops
