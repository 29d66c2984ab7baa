// Which tile takes a product or the weight gradients, how their sums are cut, and what of their work memory holds what: from sizes alone, without HIP.
#pragma once
#include <stdint.h>

#include <algorithm>

#include "op_sizes.h"

namespace cams_ops {

constexpr int kProductStep = 64;         // bytes of k in a stage of LDS
constexpr int kWeightStep = 32;          // rows in a stage of LDS
constexpr int kBiasCols = 256;           // columns whose sums over dy's rows a workgroup takes

// --- products -----------------------------------------------------------------------------------------------------------

// What a tile costs, for the choice among them: us of a step of `alone` for the first workgroup of a compute unit and of `more` for each
// that it takes besides, and `start` steps for its start and end (results of large tiles leave while nothing else runs on the unit).  Fitted to
// kernels timed over 25 sizes of products (their weights from memory, as a model's layers in turn find them) and 15 of weight gradients, from
// 16 x 4096 x 4096 to 4096 x 4096 x 4096.  There the choice was within 20 % of the best, where one tile for all would be up to 4 times off.
struct TileCost {
    int high, wide;
    double alone, more;
    int start;
    bool splits;             // whether the sum may be cut into pieces
};
constexpr int64_t kLeastPiece = 16;
// tiles of `pieces` pieces of `steps` steps; cells: of the result; bytes: of the operands.  Pieces have to gain a twentieth: the host
// pays for another launch.
inline double tile_cost(const TileCost &t, int64_t tiles, int64_t pieces, int64_t steps, double cells, double bytes)
{
    const double deep = (double)ceil_div(std::max<int64_t>(tiles * pieces, 1), 256);
    const double us = std::max((t.alone + (deep - 1) * t.more) * (double)(steps + t.start), bytes / 5e6);
    return pieces > 1 ? 1.05 * (us + 4.5 + (double)(pieces + 1) * cells * 4.0 / 3e6) : us;
}
// The least of them: f(tile, pieces, steps of a piece) for each that is cheaper than those before.
template <int kTiles, typename F>
void choose_tile(const TileCost (&costs)[kTiles], int64_t steps, double cells, double bytes, int64_t high, int64_t wide, int64_t sets, F &&f)
{
    double best = -1;
    for (const TileCost &t : costs)
        for (int64_t pieces = 1; pieces <= (t.splits ? 16 : 1); pieces *= 2) {
            const int64_t length = ceil_div(steps, pieces);
            if (pieces > 1 && length < kLeastPiece) break;
            const double us = tile_cost(t, ceil_div(high, t.high) * ceil_div(wide, t.wide) * sets, ceil_div(steps, length), length, cells, bytes);
            if (best >= 0 && us >= best) continue;
            best = us;
            f(t, ceil_div(steps, length), length);
        }
}
constexpr TileCost kProductTiles[] = {{256, 256, 1.05, 1.05, 8, false}, {256, 128, 0.65, 0.63, 7, false}, {128, 128, 0.42, 0.32, 6, true},
                                      {64, 128, 0.37, 0.20, 6, false}, {64, 64, 0.22, 0.15, 6, true}};
// Tokens up to which a product goes to product8_few, and with up to how many weights twice as many do: 32 x 4096 x 4096 9.4 us against 12.0 by tiles,
// 32 x 8192 x 8192 28.9 against 20.3.
constexpr int64_t kFewRows = 16, kFewWeights = (int64_t)1 << 25;

// Which kernel takes a product, into how many pieces k is cut, and where the work memory holds what.
struct ProductShape {
    int few;                 // tokens in sixteens for product8_few, or 0
    int high, wide;          // tokens and channels of a tile
    int splits, k_split;
    int64_t tiles_m, tiles_n, ld;
    uint64_t x_at, w_at, sums_at, bytes;
};
inline ProductShape product_shape(int64_t rows, int64_t cols, int64_t outs, bool x_aligned, bool w_aligned)
{
    ProductShape s = {};
    s.splits = 1;
    if (rows <= kFewRows || (rows <= 2 * kFewRows && outs * cols <= kFewWeights)) {
        s.few = rows <= kFewRows ? 1 : 2;
        s.tiles_m = 1, s.tiles_n = ceil_div(outs, 16);
        return s;
    }
    choose_tile(kProductTiles, ceil_div(std::max<int64_t>(cols, 1), kProductStep), (double)rows * (double)outs, (double)cols * (double)(rows + outs), rows, outs, 1,
                [&](const TileCost &t, int64_t pieces, int64_t length) {
                    s.high = t.high, s.wide = t.wide, s.tiles_m = ceil_div(rows, t.high), s.tiles_n = ceil_div(outs, t.wide);
                    s.k_split = (int)(length * kProductStep), s.splits = (int)pieces;
                });
    s.ld = ceil_div(cols, 16) * 16;
    if (cols % 16) x_aligned = w_aligned = false;
    s.x_at = 0;
    s.w_at = s.x_at + (x_aligned ? 0 : (uint64_t)(rows * s.ld));
    s.sums_at = s.w_at + (w_aligned ? 0 : (uint64_t)(outs * s.ld));
    s.bytes = s.sums_at + (s.splits > 1 ? (uint64_t)s.splits * (uint64_t)rows * (uint64_t)outs * sizeof(int32_t) : 0);
    return s;
}

// --- weight gradients --------------------------------------------------------------------------------------------------

constexpr int64_t kMostChannels = (int64_t)1 << 23;      // a step's rows lie within 31 bits

constexpr TileCost kWeightTiles[] = {{256, 256, 0.83, 0.83, 16, false}, {128, 128, 0.32, 0.24, 6, true}, {64, 64, 0.16, 0.11, 6, true}};

// How a call is cut, and where its work memory holds what.
struct WeightShape {
    int tile;                // input and output channels of a tile
    int q_planes, dy_planes; // one of them is 1
    bool copied;             // dy is written anew
    int64_t tiles_i, tiles_o;
    int64_t splits, split_steps;         // pieces of the sum over planes and steps of rows, steps of a piece
    int64_t bias_chunks, bias_rows;      // pieces of a worker's rows for the bias, rows of a piece
    int64_t a_ld, b_ld;
    uint64_t a_at, b_at, sums_at, bias_at, bytes;
};
// wide: the gradients are fp32.  Scales of powers of two leave dy its bits: 8, or 11 in two planes.
inline WeightShape weight_shape(int64_t rows, int64_t cols, int64_t outs, int32_t n, bool binary, int32_t type, bool dy_aligned, bool wide)
{
    const int64_t per = rows / n;
    WeightShape s = {};
    const bool as_it_lies = dy_aligned && outs % 8 == 0;
    s.q_planes = 1;
    const int planes = type == COMP_AMS_F32 ? 3 : binary ? (type == COMP_AMS_F16 ? 2 : 1) : wide ? 3 : 2;
    s.dy_planes = planes;
    // bytes written: planes of q scale, and dy if it is not read as it lies; or q and planes of dy scale
    if (type == COMP_AMS_BF16 && !binary && planes * cols + (as_it_lies ? 0 : outs) <= cols + planes * outs) s.q_planes = planes, s.dy_planes = 1;
    s.copied = s.dy_planes > 1 || !as_it_lies;
    const int64_t steps = std::max<int64_t>(1, ceil_div(per, kWeightStep) * s.q_planes * s.dy_planes);
    choose_tile(kWeightTiles, steps, (double)cols * (double)outs * n, 0.0, cols, outs, n, [&](const TileCost &t, int64_t pieces, int64_t length) {
        s.tile = t.high, s.tiles_i = ceil_div(cols, t.high), s.tiles_o = ceil_div(outs, t.wide);
        s.split_steps = length, s.splits = pieces;
    });
    const int64_t want = std::max<int64_t>(1, 1024 / (n * ceil_div(std::max<int64_t>(outs, 1), kBiasCols)));
    s.bias_rows = std::max<int64_t>(64, ceil_div(per, want));
    s.bias_chunks = std::max<int64_t>(1, ceil_div(per, s.bias_rows));
    s.a_ld = ceil_div(cols, 8) * 8, s.b_ld = ceil_div(outs, 8) * 8;
    const uint64_t a_bytes = (uint64_t)(s.q_planes * rows * s.a_ld) * 2, b_bytes = s.copied ? (uint64_t)(s.dy_planes * rows * s.b_ld) * 2 : 0;
    const uint64_t sums = s.splits > 1 ? (uint64_t)(s.splits * n) * (uint64_t)(cols * outs) * sizeof(float) : 0;
    s.a_at = 0;
    s.b_at = s.a_at + a_bytes;
    s.sums_at = s.b_at + b_bytes;
    s.bias_at = s.sums_at + (sums + 15) / 16 * 16;
    s.bytes = s.bias_at + (uint64_t)(s.bias_chunks * n * outs) * sizeof(float);
    return s;
}

}  // namespace cams_ops
