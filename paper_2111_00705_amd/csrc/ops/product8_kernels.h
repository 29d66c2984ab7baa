// Product of 8-bit integers with a scale for each token and channel.
//
//   y[m][n] = (sum_k x[m][k] w[n][k]) x_scale[m] w_scale[n] + bias[n]
//
// The sums are 32-bit integers and exact in any order (fewer than 2^17 products of at most 2^14).
// Both operands lie along k, so a tile's rows go to LDS as they are.  The matrix instruction takes the channels as its rows: a lane then holds
// four neighbouring channels of one token.
//
// 16384 x 4096 x 4096 to bfloat16 takes 222 to 235 us by the card, 2470 TOP/s at best: bound by power.  The matrix units are busy 59 % of the time at a clock that falls from 2.0
// to 1.7 GHz as that share rises, so what was left to gain was energy and the time that results take: read from LDS between barriers, two stages, results
// stored as they are held, it took 309 us; four stages and fragments a step ahead 5 % less; results through LDS in whole lines and past the caches
// 222.  The instruction of 32 x 32 results in place of 16 x 16 took 20 % more, four wavefronts of 128 x 128 in place of eight of 128 x 64 a quarter more.
// Few tokens are bound by the weights' bytes and by latency: 4 x 4096 x 4096 5.5 us alone (3.0 TB/s), 4 x 8192 x 8192 16 (4.2).
// Short sums are bound by each tile's first load and its end, which waits for no load since scales and bias come to LDS before the sum:
// 16384 x 64 x 4096 40 us (48 before), 14704 x 576 x 2304 38 (43), where the results alone are 22 and 11.
#pragma once
#include "rows8.h"
#include "rows8_shapes.h"

namespace cams_ops {

typedef int v4i __attribute__((ext_vector_type(4)));

struct ProductArgs {
    int64_t rows, outs, x_stride, w_stride, y_stride;
    int cols;                    // k
    int tiles_m, tiles_n;
    int splits, k_split;         // pieces of k and their length, a multiple of kProductStep
    unsigned first;
    bool stream_out;             // y is stored as a stream
};

constexpr int kXcds = 8;

// Memory to LDS without registers, asynchronous: a lane's 16 bytes at `offset` of a buffer (base, size in bytes; zeros from its end on) go to `to` +
// 16 lane, `to` and the buffer being the wavefront's.  vmcnt counts it.  In assembly, because the compiler takes every read of LDS for one of
// what is still on its way and waits for memory before it; there is no output that it could take for written.  The place in LDS is m0, which the
// compiler sets.
__device__ __forceinline__ v4u raw_buffer(const void *base, uint32_t bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    return v4u{(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, bytes, 0x00020000u};
}
__device__ __forceinline__ void to_lds(const v4u &buffer, uint32_t offset, const int8_t *to)
{
    const uint32_t lds = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) int8_t *)to;
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(buffer), "{m0}"(lds) : "memory");
}

// The same of 64 numbers of 32 bits.
__device__ __forceinline__ void words_to_lds(const v4u &buffer, uint32_t offset, const float *to)
{
    const uint32_t lds = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) float *)to;
    asm volatile("s_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(offset), "s"(buffer), "{m0}"(lds) : "memory");
}

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

// Sixteen rows of kFrags fragments each from a wavefront to memory: a lane holds columns 16 f + 4 (lane / 16) + 0..3 of row lane % 16.  Through the
// wavefront's own piece of LDS, so that a store takes 16 neighbouring bytes a lane and whole lines a row: stored as they are held, in
// pieces of 8 bytes, the 134 MB of 16384 x 4096 results took 110 us of 330.
// rows, cols: how many there are from the first on.
typedef float v4f __attribute__((ext_vector_type(4)));

template <typename Y, int kFrags> constexpr int kSixteenLd = kFrags * 16 + 16 / (int)sizeof(Y);       // elements from row to row in LDS
template <typename Y, int kFrags>
__device__ __forceinline__ void store_sixteen(Y *lds, const Y (&v)[kFrags][4], Y *to, int64_t stride, int64_t rows, int64_t cols, bool stream)
{
    constexpr int E = 16 / (int)sizeof(Y), kLd = kSixteenLd<Y, kFrags>, kLanes = kFrags * 16 / E, kRows = kWave / kLanes;
    const int lane = threadIdx.x % kWave;
    Y *mine = lds + (lane & 15) * kLd + (lane >> 4) * 4;
#pragma unroll
    for (int f = 0; f < kFrags; ++f) {
        if constexpr (sizeof(Y) == 4) *reinterpret_cast<v4u *>(mine + f * 16) = v4u{bits1(v[f][0]), bits1(v[f][1]), bits1(v[f][2]), bits1(v[f][3])};
        else *reinterpret_cast<uint64_t *>(mine + f * 16) = (uint64_t)(bits1(v[f][2]) | (bits1(v[f][3]) << 16)) << 32 | (bits1(v[f][0]) | (bits1(v[f][1]) << 16));
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const int col = lane % kLanes * E;
#pragma unroll
    for (int r = 0; r < 16; r += kRows) {
        const int row = r + lane / kLanes;
        const v4u raw = *reinterpret_cast<const v4u *>(lds + row * kLd + col);
        if (row >= rows || col >= cols) continue;
        Y *p = to + row * stride + col;
        if (col + E <= cols) {
            store_vec(p, raw, stream);
        } else {
#pragma unroll
            for (int q = 0; q < E; ++q) {
                const uint32_t bits = sizeof(Y) == 4 ? raw[q * (int)sizeof(Y) / 4] : raw[q / 2] >> (16 * (q & 1));
                if (col + q < cols) {
                    if constexpr (sizeof(Y) == 4) reinterpret_cast<uint32_t *>(p)[q] = bits;
                    else reinterpret_cast<uint16_t *>(p)[q] = (uint16_t)bits;
                }
            }
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
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

constexpr int kPackThreads = 256;

struct PackArgs {
    int64_t rows, outs, x_stride, w_stride, ld;      // ld: cols rounded up to 16
    int cols, lanes;                                 // lanes that share a row, a power of two up to kPackThreads
    unsigned blocks_x;                               // workgroups for x; the others are for w
    unsigned first;
};

// Rows of x and of w written anew, 16 bytes by 16 bytes, zeros behind the row: what product8 takes, from rows of any length, stride and address.
static __global__ __launch_bounds__(kPackThreads) void product8_pack(int8_t *__restrict__ x_out, int8_t *__restrict__ w_out, const int8_t *__restrict__ x,
                                                                     const int8_t *__restrict__ w, PackArgs a)
{
    unsigned block = a.first + blockIdx.x;
    const bool of_x = block < a.blocks_x;
    if (!of_x) block -= a.blocks_x;
    const int64_t row = (int64_t)block * (kPackThreads / a.lanes) + threadIdx.x / a.lanes;
    if (row >= (of_x ? a.rows : a.outs)) return;
    const int8_t *from = of_x ? x + row * a.x_stride : w + row * a.w_stride;
    int8_t *to = (of_x ? x_out : w_out) + row * a.ld;
    for (int k = threadIdx.x % a.lanes * 16; k < a.cols; k += a.lanes * 16) *reinterpret_cast<v4i *>(to + k) = load_row16(from, k, a.cols);
}

template <int kM, int kN> constexpr int kProductStages = kM + kN <= 128 ? 8 : 4;

// A tile of kM tokens x kN channels by kWavesM x kWavesN wavefronts.  Rows, strides and addresses are multiples of 16 bytes: memory goes to LDS
// without registers.  kSplit: a piece of k; the sums go to work[piece][rows][outs].
//
// A step is 64 bytes of k.  Of the stages in LDS one has arrived and is read into registers while the matrix instructions work on what was read
// before, and the others but one are on their way from memory: one barrier a step, and nothing waits for memory or LDS within it.  Four stages fill the
// LDS for tiles of 256 x 256; those of 64 x 64, whose steps are shorter than memory takes for three, have eight.  A step's row is four
// 16-byte chunks; chunk c of row r stands at place c ^ (r / 2 & 3), so that eight rows at one chunk lie in different banks.
template <typename Y, int kM, int kN, int kWavesM, int kWavesN, bool kSplit>
__global__ __launch_bounds__(kWavesM *kWavesN *kWave, 2) void product8(Y *__restrict__ y, int *__restrict__ work, const int8_t *__restrict__ x,
                                                                    const float *__restrict__ x_scale, const int8_t *__restrict__ w,
                                                                    const float *__restrict__ w_scale, const float *__restrict__ bias,
                                                                    ProductArgs a)
{
    constexpr int kWaves = kWavesM * kWavesN, kRows = kM + kN, kStep = kProductStep, kStages = kProductStages<kM, kN>;
    constexpr int kMi = kM / kWavesM / 16, kNi = kN / kWavesN / 16;
    constexpr int kLoads = kRows / 16 / kWaves, kLoadsX = kM / 16 / kWaves;     // wavefront-wide loads of 16 rows each
    static_assert(kM % (16 * kWaves) == 0 && kN % (16 * kWaves) == 0, "whole loads");
    __shared__ __attribute__((aligned(1024))) int8_t tile[kStages][kRows * kStep];
    __shared__ __attribute__((aligned(16))) float factors[kSplit ? 1 : kM + 2 * kN];        // scales of the tokens, of the channels, and the bias

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const unsigned block = a.first + blockIdx.x;
    int piece, tm, tn;
    grouped_tile(block, (unsigned)a.splits, a.tiles_m, a.tiles_n, piece, tm, tn);
    const int64_t m0 = (int64_t)tm * kM, n0 = (int64_t)tn * kN;
    const int rows_m = (int)min((int64_t)kM, a.rows - m0), rows_n = (int)min((int64_t)kN, a.outs - n0);
    const int k_begin = kSplit ? piece * a.k_split : 0, k_end = kSplit ? min(a.cols, k_begin + a.k_split) : a.cols;
    const int8_t *xt = x + m0 * a.x_stride, *wt = w + n0 * a.w_stride;

    // a lane's part of each load: row lane / 4 of the sixteen, the chunk that belongs to place lane % 4
    const int chunk = (lane & 3) ^ ((lane >> 3) & 3);
    constexpr uint32_t kNowhere = 0x80000000u;       // past the end of any tile: reads zeros
    uint32_t off[kLoads];
    const v4u xsrc = raw_buffer(xt, 0x7fffffff), wsrc = raw_buffer(wt, 0x7fffffff);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const bool of_x = j < kLoadsX;
        const int row = ((of_x ? j : j - kLoadsX) * kWaves + wave) * 16 + (lane >> 2);
        off[j] = row < (of_x ? rows_m : rows_n) ? (uint32_t)(row * (of_x ? a.x_stride : a.w_stride) + chunk * 16 + k_begin) : kNowhere;
    }
    auto place = [&](int j) {                        // first byte in LDS of load j
        return ((j < kLoadsX ? j * kWaves : kM / 16 + (j - kLoadsX) * kWaves) + wave) * 1024;
    };
    int k_next = k_begin;
    auto send = [&](int stage) {                     // the next step, memory to LDS, asynchronous
        const bool whole = k_next + kStep <= k_end;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            uint32_t at = off[j];
            if (!whole && k_next + chunk * 16 >= k_end) at = kNowhere;
            to_lds(j < kLoadsX ? xsrc : wsrc, at, &tile[stage][place(j)]);
            off[j] += kStep;
        }
        k_next += kStep;
    };

    v4i acc[kNi][kMi];
#pragma unroll
    for (int n = 0; n < kNi; ++n)
#pragma unroll
        for (int m = 0; m < kMi; ++m) acc[n][m] = v4i{0, 0, 0, 0};
    const int wm = wave / kWavesN, wn = wave % kWavesN;
    const int frow = lane & 15, fgroup = lane >> 4;
    const int fat = frow * kStep + (fgroup ^ ((frow >> 1) & 3)) * 16;
    struct Frags {
        v4i w[kNi], x[kMi];
    };
    auto read = [&](Frags &f, int stage) {
        const int8_t *xs = &tile[stage][wm * kMi * 16 * kStep + fat];
        const int8_t *ws = &tile[stage][(kM + wn * kNi * 16) * kStep + fat];
#pragma unroll
        for (int n = 0; n < kNi; ++n) f.w[n] = *reinterpret_cast<const v4i *>(ws + n * 16 * kStep);
#pragma unroll
        for (int m = 0; m < kMi; ++m) f.x[m] = *reinterpret_cast<const v4i *>(xs + m * 16 * kStep);
    };
    auto multiply = [&](const Frags &f) {
#pragma unroll
        for (int m = 0; m < kMi; ++m)
#pragma unroll
            for (int n = 0; n < kNi; ++n) acc[n][m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f.w[n], f.x[m], acc[n][m], 0, 0, 0);
    };
    constexpr int kPer = kMi * kNi / (kMi + kNi);
    auto mixed = [&]() {
#pragma unroll
        for (int u = 0; u < kMi + kNi; ++u) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);          // a read from LDS
            __builtin_amdgcn_sched_group_barrier(0x008, kPer, 0);       // matrix instructions
        }
        __builtin_amdgcn_sched_group_barrier(0x008, kMi * kNi - kPer * (kMi + kNi), 0);
    };
    // One step: the next stage has arrived, for every wavefront (those sent after it may still be on their way), and nobody reads the one before
    // any more, which the youngest step takes.  Steps past the end read zeros.
    auto step = [&](int u, const Frags &now, Frags &next) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((kStages - 3) * kLoads) : "memory");
        send((u + kStages - 1) % kStages);
        read(next, (u + 1) % kStages);
        multiply(now);
        mixed();
    };
    Frags even, odd;
    const int steps = (k_end - k_begin + kStep - 1) / kStep;
    if constexpr (!kSplit) {                         // before all others, and so there before any of them: at the end nothing waits for memory
        const v4u from[3] = {raw_buffer(x_scale + m0, (uint32_t)rows_m * 4u), raw_buffer(w_scale + n0, (uint32_t)rows_n * 4u),
                             raw_buffer(bias ? bias + n0 : bias, bias ? (uint32_t)rows_n * 4u : 0u)};
        constexpr int kOfX = kM / kWave, kOfN = kN / kWave;
#pragma unroll
        for (int j = 0; j < kOfX + 2 * kOfN; ++j) {
            const int which = j < kOfX ? 0 : j < kOfX + kOfN ? 1 : 2, part = j - (which == 0 ? 0 : which == 1 ? kOfX : kOfX + kOfN);
            if (wave == j % kWaves) words_to_lds(from[which], (uint32_t)(part * kWave + lane) * 4u, &factors[j * kWave]);
        }
    }
#pragma unroll
    for (int u = 0; u < kStages - 1; ++u) send(u);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((kStages - 2) * kLoads) : "memory");
    read(even, 0);
    int s = 0;
    for (; s + kStages <= steps; s += kStages) {
#pragma unroll
        for (int u = 0; u < kStages; u += 2) {
            step(u, even, odd);
            step(u + 1, odd, even);
        }
    }
#pragma unroll
    for (int u = 0; u < kStages; u += 2) {           // the last ones, in pairs
        if (s + u >= steps) break;
        step(u, even, odd);
        step(u + 1, odd, even);
    }
    if constexpr (kSplit) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");     // LDS belongs to the next workgroup after this one
#pragma unroll
        for (int n = 0; n < kNi; ++n)
#pragma unroll
            for (int m = 0; m < kMi; ++m) {
                const int64_t at_n = n0 + (wn * kNi + n) * 16 + fgroup * 4, at_m = m0 + (wm * kMi + m) * 16 + frow;
                if (at_m >= a.rows || at_n >= a.outs) continue;
                int *p = work + ((int64_t)piece * a.rows + at_m) * a.outs + at_n;
                if (at_n + 4 <= a.outs) {
                    *reinterpret_cast<v4u_any *>(p) = __builtin_bit_cast(v4u, acc[n][m]);
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (at_n + q < a.outs) p[q] = acc[n][m][q];
                }
            }
    } else {
        // nothing is on its way to LDS or read from it any more, by any wavefront
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        float ws[kNi][4], b[kNi][4], xs[kMi];
#pragma unroll
        for (int n = 0; n < kNi; ++n) {
            const float *at = &factors[kM + (wn * kNi + n) * 16 + fgroup * 4];
            *reinterpret_cast<v4f *>(ws[n]) = *reinterpret_cast<const v4f *>(at);
            *reinterpret_cast<v4f *>(b[n]) = *reinterpret_cast<const v4f *>(at + kN);
        }
#pragma unroll
        for (int m = 0; m < kMi; ++m) xs[m] = factors[(wm * kMi + m) * 16 + frow];
        Y *mine = reinterpret_cast<Y *>(&tile[0][0]) + wave * 16 * kSixteenLd<Y, kNi>;
        static_assert(kWaves * 16 * kSixteenLd<Y, kNi> * sizeof(Y) <= sizeof tile, "room for the results");
#pragma unroll
        for (int m = 0; m < kMi; ++m) {
            Y out[kNi][4];
#pragma unroll
            for (int n = 0; n < kNi; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q) out[n][q] = narrow1<Y>((float)acc[n][m][q] * xs[m] * ws[n][q] + b[n][q]);
            const int64_t at_m = m0 + (wm * kMi + m) * 16, at_n = n0 + wn * kNi * 16;
            store_sixteen<Y, kNi>(mine, out, y + at_m * a.y_stride + at_n, a.y_stride, a.rows - at_m, a.outs - at_n, a.stream_out);
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
