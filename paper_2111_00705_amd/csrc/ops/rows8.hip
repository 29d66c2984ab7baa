// Host side of include/comp_ams_rows8.h: argument validation, the choice of kernels, launches.
#include "../../../include/comp_ams_rows8.h"

#include "op_host.h"

#include "product8_kernels.h"
#include "rms_kernels.h"
#include "rows8.h"
#include "rows8_shapes.h"
#include "weight_kernels.h"

using namespace cams_ops;

namespace {

// Rows of int8: any alignment.
#define REQUIRE_BYTE_ROWS(what, name, p, rows, cols, stride)                                                                   \
    do {                                                                                                                       \
        REQUIRE((p) != nullptr || (rows) == 0 || (cols) == 0, "%s: %s is NULL", what, name);                                   \
        REQUIRE((stride) >= (cols) || (rows) <= 1, "%s: the rows of %s overlap (stride %lld < %lld)", what, name,              \
                (long long)(stride), (long long)(cols));                                                                       \
        REQUIRE((stride) >= 0 && ((rows) <= 1 || (stride) < kMaxElements / (rows)), "%s: %s is out of range", what, name);     \
    } while (0)

constexpr int64_t kLimit31 = (int64_t)1 << 31;
constexpr int64_t kMostStride = kLimit31 / 512;      // bytes between rows, of which a tile has 256

// Whether a product's result is stored past the caches: only rows that begin at multiples of 128 bytes.  Lines that two tiles share have to meet in a
// cache: weight gradients of 4 workers' 128 rows, 4096 x 4096, past the caches / through them, at such rows 47 / 51 us, 20 bytes further 86 / 53.
bool streamed_result(const void *p, int64_t elements, int64_t row_stride, int64_t set_stride, int32_t type)
{
    const int64_t size = (int64_t)type_size(type);
    return streamed_out(elements, type) && aligned(p, 128) && row_stride * size % 128 == 0 && set_stride * size % 128 == 0;
}

// Lanes of a workgroup of 256 that share a row of `chunks`, when it is written anew.
int shared_lanes(int64_t chunks)
{
    int lanes = 8;
    while (lanes < 256 && lanes < chunks) lanes *= 2;
    return lanes;
}

// f(Shape) for the team and the vectors a lane that hold a row of `len` elements, if one does: up to kMost vectors.  Two workgroups of 512 share a
// compute unit where one of 1024 has it for itself: us by two vectors of 1024 lanes / by three or four of 512: norm 3262 x 9728 f16 45 / 29, 4000 x 16000
// bf16 with residual 104 / 86, in 8 bits and back 5853 x 8704 121 / 88, its backward pass 5000 x 10240 111 / 105.  Longer rows: the forms that read a
// row several times / three or four vectors of 1024 lanes, 5000 x 12000 fp32: norm 393 / 167, in 8 bits 456 / 164, its backward pass 425 / 191, a
// checkpoint written and read 249 / 95.
template <typename T, int kMost, typename F>
bool with_rows(int64_t len, F &&f)
{
    const int64_t vecs = ceil_div(len, kVec<T>);
    if (len < kVec<T> || vecs > kMost) return false;
    if (vecs <= 32) with_vecs<16, 1, 2>((int)ceil_div(vecs, 16), f);
    else if (vecs <= 256) with_vecs<64, 1, 4>((int)ceil_div(vecs, 64), f);
    else if (vecs <= 1024) with_vecs<256, 2, 4>((int)ceil_div(vecs, 256), f);
    else if (vecs <= 2048) with_vecs<512, 3, 4>((int)ceil_div(vecs, 512), f);
    else if constexpr (kMost > 2048) with_vecs<1024, 3, 4>((int)ceil_div(vecs, 1024), f);
    return true;
}

int rows8_check(const char *what, int64_t rows, int64_t cols, const float *scale, int32_t type)
{
    REQUIRE(known_type(type), "%s: unknown type %d", what, type);
    REQUIRE(rows >= 0 && rows < kLimit31, "%s: rows=%lld must be in [0, 2^31)", what, (long long)rows);
    REQUIRE(cols >= 0 && cols < kLimit31, "%s: cols=%lld must be in [0, 2^31)", what, (long long)cols);
    REQUIRE(scale || rows == 0, "%s: scale is NULL", what);
    REQUIRE(aligned(scale, 4), "%s: scale must be 4-byte aligned", what);
    return COMP_AMS_OK;
}

// --- the norm --------------------------------------------------------------------------------------------------------

int rms_check(const char *what, int64_t rows, int64_t cols, int32_t type)
{
    REQUIRE(known_type(type), "%s: unknown type %d", what, type);
    REQUIRE(rows >= 0 && rows < (int64_t)1 << 40, "%s: rows=%lld must be in [0, 2^40)", what, (long long)rows);
    REQUIRE(cols >= 1 && cols < kLimit31, "%s: cols=%lld must be in [1, 2^31)", what, (long long)cols);
    return COMP_AMS_OK;
}

// Workgroups of the forward pass, us at 1024 / 2048 / 4096: in 8 bits 16384 x 2048 bf16 47.5 / 45.4 / 43.0; 8192 x 4096 bf16 48.7 / 50.4 / 47.9;
// 16384 x 768 19.4 / 20.4 / 20.7.
constexpr int64_t kRmsBlocks = 4096;
// Workgroups that the rows of all workers are cut into in the backward pass.  More keep more rows in flight, and write
// more partial sums.  us with the join, at 512 / 750 / 1024 / 2048: 16384 x 768 bf16, n = 8 22.4 / 23.8 / 21.6 / 24.8; 20000 x 2047 fp32 kept in 8 bits,
// n = 20 134 / 129 / 117 / 118; 8192 x 4096 bf16, n = 4 67.8 / 66.1 / 67.2 / 73.9.
constexpr int64_t kRmsChunkBlocks = 1024;

// How a worker's rows are cut for the gain's gradients: chunks of rows with one set of column sums each.
struct RmsChunks {
    int64_t rows, count;     // rows of a chunk; chunks of a worker
};
// A workgroup takes as many rows at a time as it has teams (of fp32 rows; 16-bit rows have a team for twice the columns): one such turn where rows
// are few, four at least where they fill the chip.  us at 4 / 2 / 1 turns: 1024 x 4096 bf16, n = 8 15.6 / 16.5 / 23.2; 64 x 8192, n = 2 17.2 / - / 12.3.
// Up to two turns of a worker's rows are one chunk, which needs no join and no launch for it.
RmsChunks rms_chunks(int64_t worker_rows, int64_t cols, int32_t n)
{
    const int64_t teams = cols <= 128 ? 16 : cols <= 1024 ? 4 : 1;
    if (worker_rows <= 2 * teams) return {2 * teams, 1};
    const int64_t turns = std::min<int64_t>(4, ceil_div(worker_rows * n, 256 * teams));
    const int64_t want = std::max<int64_t>(1, ceil_div(kRmsChunkBlocks, n));
    const int64_t rows = std::max<int64_t>(turns * teams, ceil_div(worker_rows, want));
    return {rows, std::max<int64_t>(1, ceil_div(worker_rows, rows))};
}

// Rows that are read once, from memory: loads that do not stay in the caches.  us with the caches / past them: backward 8192 x 4096 bf16 67.6 / 58.5,
// forward in 8 bits 16384 x 2048 42.4 / 40.0; 16384 x 768, which the memory-side cache holds, 16.5 / 19.8 forward.
bool streamed_rows(int64_t elements, int32_t type) { return elements > ((int64_t)48 << 20) / (int64_t)type_size(type); }
// h is read again by the norm after the next product, when little of it would be left in the caches.
bool streamed_h(int64_t elements, int32_t type) { return elements > ((int64_t)16 << 20) / (int64_t)type_size(type); }

int rms_forward_call(const char *what, void *y, float *scale, void *h, float *rstd, const void *x, const void *residual, const float *gain,
                     const RmsArgs &a, bool q8, int32_t type, hipStream_t stream)
{
    if (a.rows == 0) return COMP_AMS_OK;
    with_type(type, [&](auto t) {
        using T = decltype(t);
        auto call = [&](auto eight) {
            constexpr bool k8 = decltype(eight)::value;
            const bool held = with_rows<T, 4096>(a.cols, [&](auto shape) {
                using S = decltype(shape);
                const int64_t teams = kTeamBlock<S::threads> / S::threads;
                rms_forward<T, S::threads, S::vecs, k8><<<(unsigned)std::min<int64_t>(ceil_div(a.rows, teams), kRmsBlocks), kTeamBlock<S::threads>, 0, stream>>>(
                    y, scale, static_cast<T *>(h), rstd, static_cast<const T *>(x), static_cast<const T *>(residual), gain, a);
            });
            if (!held)
                rms_forward_any<T, k8><<<(unsigned)std::min(a.rows, most_blocks(kRmsThreads)), kRmsThreads, 0, stream>>>(
                    y, scale, static_cast<T *>(h), rstd, static_cast<const T *>(x), static_cast<const T *>(residual), gain, a);
        };
        if (q8) call(std::true_type{});
        else call(std::false_type{});
    });
    return launched(what);
}

#define REQUIRE_RMS_FORWARD(what)                                                                                              \
    do {                                                                                                                       \
        if (const int rc = rms_check(what, rows, cols, type)) return rc;                                                       \
        REQUIRE_ROWS(what, "x", x, rows, cols, x_stride, type);                                                                \
        if (residual) REQUIRE_ROWS(what, "residual", residual, rows, cols, residual_stride, type);                             \
        if (h) REQUIRE_ROWS(what, "h", h, rows, cols, h_stride, type);                                                         \
        REQUIRE(gain, "%s: gain is NULL", what);                                                                               \
        REQUIRE(aligned(gain, 4) && aligned(rstd, 4), "%s: gain and rstd must be 4-byte aligned", what);                       \
        REQUIRE(std::isfinite(eps) && eps >= 0.f, "%s: eps must be finite and not negative", what);                            \
    } while (0)

// --- the product -----------------------------------------------------------------------------------------------------

int product_check(const char *what, int64_t rows, int64_t cols, int64_t outs)
{
    REQUIRE(rows >= 0 && rows < kLimit31, "%s: rows=%lld must be in [0, 2^31)", what, (long long)rows);
    REQUIRE(outs >= 0 && outs < kLimit31, "%s: outs=%lld must be in [0, 2^31)", what, (long long)outs);
    REQUIRE(cols >= 0 && cols < COMP_AMS_MAX_Q8_COLS, "%s: cols=%lld must be in [0, %d)", what, (long long)cols, COMP_AMS_MAX_Q8_COLS);
    const ProductShape s = product_shape(rows, cols, outs, true, true);
    REQUIRE(s.tiles_m * s.tiles_n * s.splits <= kMaxBlocks, "%s: rows and outs are too many for one call", what);
    return COMP_AMS_OK;
}

// --- weight gradients --------------------------------------------------------------------------------------------------

int weight_check(const char *what, int64_t rows, int64_t cols, int64_t outs, int32_t n, int32_t binary, int32_t type)
{
    REQUIRE(known_type(type), "%s: unknown type %d", what, type);
    REQUIRE(n >= 1 && n <= 65535, "%s: n=%d must be in [1, 65535]", what, n);
    REQUIRE(rows >= 0 && rows < (int64_t)1 << 32 && rows / n < kLimit31 / 4, "%s: rows=%lld are too many", what, (long long)rows);
    REQUIRE(rows % n == 0, "%s: rows=%lld must be a multiple of n=%d", what, (long long)rows, n);
    REQUIRE(cols >= 0 && cols <= kMostChannels && outs >= 0 && outs <= kMostChannels, "%s: cols=%lld or outs=%lld is out of range", what,
            (long long)cols, (long long)outs);
    for (bool wide : {false, true}) {
        const WeightShape s = weight_shape(rows, cols, outs, n, binary != 0, type, true, wide);
        REQUIRE(s.tiles_i * s.tiles_o <= kMaxBlocks / n / s.splits, "%s: cols, outs and n are too many for one call", what);
    }
    return COMP_AMS_OK;
}

// Rows in bfloat16 for the product (if there is one), and the sums of dy's columns (if there is a bias).
void weight_prepare_launch(const WeightShape &s, char *work, const void *dy, const int8_t *q, const float *scale, int64_t rows, int64_t cols,
                           int64_t outs, int64_t dy_stride, int64_t q_stride, int32_t n, bool binary, bool bias, int32_t type, hipStream_t stream)
{
    PrepareArgs a = {};
    a.rows = rows, a.cols = cols, a.outs = outs, a.q_stride = q_stride, a.dy_stride = dy_stride;
    a.a_ld = s.a_ld, a.b_ld = s.b_ld, a.a_plane = rows * s.a_ld, a.b_plane = rows * s.b_ld;
    a.worker_rows = rows / n, a.bias_rows = s.bias_rows, a.bias_chunks = (unsigned)s.bias_chunks;
    a.lanes_a = shared_lanes(s.a_ld / 8), a.lanes_b = shared_lanes(s.b_ld / 8);
    const bool product = rows > 0 && cols > 0;
    a.blocks_a = product ? (unsigned)ceil_div(rows, kPrepareThreads / a.lanes_a * kPrepareRows) : 0u;
    a.blocks_b = product && s.copied ? (unsigned)ceil_div(rows, kPrepareThreads / a.lanes_b * kPrepareRows) : 0u;
    const int64_t blocks = (int64_t)a.blocks_a + a.blocks_b + (bias ? n * s.bias_chunks * ceil_div(outs, kBiasCols) : 0);
    auto go = [&](auto t, auto q_planes, auto dy_planes) {
        using T = decltype(t);
        constexpr int kQ = decltype(q_planes)::value, kD = decltype(dy_planes)::value;
        auto launch = [&](auto kernel) {
            in_launches(blocks, kPrepareThreads, [&](unsigned first, unsigned count) {
                a.first = first;
                kernel<<<count, kPrepareThreads, 0, stream>>>(reinterpret_cast<bf16_t *>(work + s.a_at), reinterpret_cast<bf16_t *>(work + s.b_at),
                                                              reinterpret_cast<float *>(work + s.bias_at), static_cast<const T *>(dy), q, scale, a);
            });
        };
        if (bias) launch(weight_prepare<T, kQ, kD, true>);
        else launch(weight_prepare<T, kQ, kD, false>);
    };
    constexpr std::integral_constant<int, 1> one{};
    constexpr std::integral_constant<int, 2> two{};
    constexpr std::integral_constant<int, 3> three{};
    if (type == COMP_AMS_F32) go(float{}, one, three);
    else if (type == COMP_AMS_F16 && s.dy_planes == 3) go(f16_t{}, one, three);
    else if (type == COMP_AMS_F16) go(f16_t{}, one, two);
    else if (s.q_planes == 3) go(bf16_t{}, three, one);
    else if (s.q_planes == 2) go(bf16_t{}, two, one);
    else if (s.dy_planes == 3) go(bf16_t{}, one, three);
    else if (s.dy_planes == 2) go(bf16_t{}, one, two);
    else go(bf16_t{}, one, one);
}

template <typename G>
void weight_launch(G *out, G *dbias, const bf16_t *a_rows, const bf16_t *b_rows, const float *bias_sums, WeightArgs a, int tile, bool in_first,
                   hipStream_t stream)
{
    const int64_t tiles = (int64_t)a.tiles_i * a.tiles_o * a.n * a.splits;
    a.tiles = (unsigned)tiles;
    auto go = [&](auto kernel, int threads) {
        in_launches(tiles + (dbias ? a.n * ceil_div(a.outs, threads) : 0), threads, [&](unsigned first, unsigned count) {
            a.first = first;
            kernel<<<count, threads, 0, stream>>>(out, dbias, a_rows, b_rows, bias_sums, a);
        });
    };
    auto form = [&](auto first) {
        constexpr bool kFirst = decltype(first)::value;
        if (tile == 256) go(weight_grad<G, kFirst, 256, 256, 2, 4>, 512);
        else if (tile == 128) go(weight_grad<G, kFirst, 128, 128, 2, 2>, 256);
        else go(weight_grad<G, kFirst, 64, 64, 2, 2>, 256);
    };
    if (in_first) form(std::true_type{});
    else form(std::false_type{});
}

}  // namespace

extern "C" {

int comp_ams_quantize_rows(int8_t *q, float *scale, const void *x, int64_t rows, int64_t cols, int64_t q_stride, int64_t x_stride,
                           int32_t binary, int32_t type, void *hip_stream)
{
    const char *what = "quantize_rows";
    if (const int rc = rows8_check(what, rows, cols, scale, type)) return rc;
    REQUIRE_BYTE_ROWS(what, "q", q, rows, cols, q_stride);
    REQUIRE_ROWS(what, "x", x, cols ? rows : 0, cols, x_stride, type);
    if (rows == 0) return COMP_AMS_OK;
    QuantArgs a = {rows, cols, x_stride, q_stride, binary != 0, streamed_in(rows * cols, type), 0};
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    with_type(type, [&](auto t) {
        using T = decltype(t);
        const bool held = with_rows<T, 4096>(cols, [&](auto shape) {
            using S = decltype(shape);
            in_launches(ceil_div(rows, kTeamBlock<S::threads> / S::threads), kTeamBlock<S::threads>, [&](unsigned first, unsigned count) {
                a.first = first;
                quantize<T, S::threads, S::vecs><<<count, kTeamBlock<S::threads>, 0, stream>>>(q, scale, static_cast<const T *>(x), a);
            });
        });
        if (!held)
            quantize_any<T><<<(unsigned)std::min(rows, most_blocks(kQuantThreads)), kQuantThreads, 0, stream>>>(q, scale, static_cast<const T *>(x), a);
    });
    return launched(what);
}

int comp_ams_restore_rows(void *x, const int8_t *q, const float *scale, int64_t rows, int64_t cols, int64_t x_stride, int64_t q_stride,
                          int32_t type, void *hip_stream)
{
    const char *what = "restore_rows";
    if (const int rc = rows8_check(what, rows, cols, scale, type)) return rc;
    REQUIRE_BYTE_ROWS(what, "q", q, rows, cols, q_stride);
    REQUIRE_ROWS(what, "x", x, cols ? rows : 0, cols, x_stride, type);
    if (rows == 0 || cols == 0) return COMP_AMS_OK;
    QuantArgs a = {rows, cols, x_stride, q_stride, false, streamed_out(rows * cols, type), 0};
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    with_type(type, [&](auto t) {
        using T = decltype(t);
        const bool held = with_rows<T, 4096>(cols, [&](auto shape) {
            using S = decltype(shape);
            in_launches(ceil_div(rows, kTeamBlock<S::threads> / S::threads), kTeamBlock<S::threads>, [&](unsigned first, unsigned count) {
                a.first = first;
                restore<T, S::threads, S::vecs><<<count, kTeamBlock<S::threads>, 0, stream>>>(static_cast<T *>(x), q, scale, a);
            });
        });
        if (!held)
            restore_any<T><<<(unsigned)std::min(rows, most_blocks(kQuantThreads)), kQuantThreads, 0, stream>>>(static_cast<T *>(x), q, scale, a);
    });
    return launched(what);
}

int comp_ams_rms_norm(void *y, void *h, float *rstd, const void *x, const void *residual, const float *gain, int64_t rows, int64_t cols,
                      int64_t y_stride, int64_t h_stride, int64_t x_stride, int64_t residual_stride, float eps, int32_t type,
                      void *hip_stream)
{
    const char *what = "rms_norm";
    REQUIRE_RMS_FORWARD(what);
    REQUIRE_ROWS(what, "y", y, rows, cols, y_stride, type);
    REQUIRE(!h || h != y || rows == 0, "%s: y and h are the same array", what);
    const RmsArgs a = {rows, cols, x_stride, residual_stride, h_stride, y_stride, eps, (float)(1.0 / (double)cols), false,
                       streamed_rows(rows * cols, type), streamed_out(rows * cols, type), streamed_h(rows * cols, type)};
    return rms_forward_call(what, y, nullptr, h, rstd, x, residual, gain, a, false, type, static_cast<hipStream_t>(hip_stream));
}

int comp_ams_rms_norm_q8(int8_t *q, float *scale, void *h, float *rstd, const void *x, const void *residual, const float *gain,
                         int64_t rows, int64_t cols, int64_t q_stride, int64_t h_stride, int64_t x_stride, int64_t residual_stride,
                         float eps, int32_t binary, int32_t type, void *hip_stream)
{
    const char *what = "rms_norm_q8";
    REQUIRE_RMS_FORWARD(what);
    REQUIRE_BYTE_ROWS(what, "q", q, rows, cols, q_stride);
    REQUIRE(scale || rows == 0, "%s: scale is NULL", what);
    REQUIRE(aligned(scale, 4), "%s: scale must be 4-byte aligned", what);
    const RmsArgs a = {rows, cols, x_stride, residual_stride, h_stride, q_stride, eps, (float)(1.0 / (double)cols), binary != 0,
                       streamed_rows(rows * cols, type), false, streamed_h(rows * cols, type)};
    return rms_forward_call(what, q, scale, h, rstd, x, residual, gain, a, true, type, static_cast<hipStream_t>(hip_stream));
}

int comp_ams_rms_norm_work_bytes(int64_t rows, int64_t cols, int32_t n, uint64_t *bytes)
{
    const char *what = "rms_norm_work_bytes";
    if (const int rc = rms_check(what, rows, cols, COMP_AMS_F32)) return rc;
    REQUIRE(n >= 1 && n <= 65535, "%s: n=%d must be in [1, 65535]", what, n);
    REQUIRE(rows % n == 0, "%s: rows=%lld must be a multiple of n=%d", what, (long long)rows, n);
    REQUIRE(bytes, "%s: bytes is NULL", what);
    *bytes = (uint64_t)rms_chunks(rows / n, cols, n).count * (uint64_t)n * (uint64_t)cols * sizeof(float);
    return COMP_AMS_OK;
}

int comp_ams_rms_norm_backward(void *dx, void *dgain, const void *dy, const void *h, const float *h_scale, const float *rstd,
                               const float *gain, const void *dresidual, int64_t rows, int64_t cols, int64_t dx_stride,
                               int64_t dy_stride, int64_t h_stride, int64_t dresidual_stride, int32_t n, int64_t grad_stride,
                               int32_t type, int32_t grad_type, void *work, uint64_t work_bytes, void *hip_stream)
{
    const char *what = "rms_norm_backward";
    if (const int rc = rms_check(what, rows, cols, type)) return rc;
    REQUIRE(known_type(grad_type), "%s: unknown gradient type %d", what, grad_type);
    REQUIRE(n >= 1 && n <= 65535, "%s: n=%d must be in [1, 65535]", what, n);
    REQUIRE(rows % n == 0, "%s: rows=%lld must be a multiple of n=%d", what, (long long)rows, n);
    if (h_scale) REQUIRE_BYTE_ROWS(what, "h", h, rows, cols, h_stride);
    else REQUIRE_ROWS(what, "h", h, rows, cols, h_stride, type);
    REQUIRE_ROWS(what, "dy", dy, rows, cols, dy_stride, type);
    REQUIRE_ROWS(what, "dx", dx, rows, cols, dx_stride, type);
    if (dresidual) REQUIRE_ROWS(what, "dresidual", dresidual, rows, cols, dresidual_stride, type);
    REQUIRE_ROWS(what, "dgain", dgain, (int64_t)n, cols, grad_stride, grad_type);
    REQUIRE(gain && (rstd || rows == 0), "%s: rstd or gain is NULL", what);
    REQUIRE(aligned(gain, 4) && aligned(rstd, 4) && aligned(h_scale, 4), "%s: rstd, gain and h_scale must be 4-byte aligned", what);
    uint64_t need = 0;
    if (const int rc = comp_ams_rms_norm_work_bytes(rows, cols, n, &need)) return rc;
    REQUIRE(work && work_bytes >= need, "%s: needs %llu bytes of work memory", what, (unsigned long long)need);
    REQUIRE(aligned(work, 16), "%s: work must be 16-byte aligned", what);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const RmsBackArgs a = {rows, cols, dx_stride, dy_stride, h_stride, dresidual_stride, (float)(1.0 / (double)cols),
                           streamed_rows(rows * cols, type), streamed_out(rows * cols, type),
                           dgain, grad_stride, grad_type};
    const RmsChunks ch = rms_chunks(rows / n, cols, n);
    float *sums = static_cast<float *>(work);
    bool held = false;
    with_type(type, [&](auto t) {
        using T = decltype(t);
        auto call = [&](auto kept) {
            using H = decltype(kept);
            const T *dyt = static_cast<const T *>(dy), *rt = static_cast<const T *>(dresidual);
            const H *ht = static_cast<const H *>(h);
            held = with_rows<T, sizeof(T) == 4 ? 4096 : 2048>(cols, [&](auto shape) {
                using S = decltype(shape);
                rms_backward<T, H, S::threads, S::vecs><<<dim3((unsigned)ch.count, (unsigned)n), kTeamBlock<S::threads>, 0, stream>>>(
                    static_cast<T *>(dx), sums, dyt, ht, h_scale, rstd, gain, rt, a, rows / n, ch.rows);
            });
            if (held) return;
            // the gain's gradients first: dx may replace dy or h
            // every launch of fewer than 2^32 threads
            in_launches(ceil_div(cols, kRmsThreads), kRmsThreads * (int)ch.count * n, [&](unsigned first, unsigned count) {
                rms_param_any<T, H><<<dim3(count, (unsigned)ch.count, (unsigned)n), kRmsThreads, 0, stream>>>(sums, dyt, ht, h_scale, rstd, a, rows / n, ch.rows,
                                                                                                             first);
            });
            if (rows > 0)
                rms_backward_any<T, H><<<(unsigned)std::min(rows, most_blocks(kRmsThreads)), kRmsThreads, 0, stream>>>(static_cast<T *>(dx), dyt, ht,
                                                                                                                      h_scale, rstd, gain, rt, a);
        };
        if (h_scale) call(int8_t{});
        else call(T{});
    });
    if (const int rc = launched(what)) return rc;              // what the join would read has not been written
    if (held && ch.count == 1) return COMP_AMS_OK;
    with_type(grad_type, [&](auto t) {
        using G = decltype(t);
        in_launches(ceil_div(cols, kColumnsJoin), kRmsThreads * n, [&](unsigned first, unsigned count) {
            columns_join<G><<<dim3(count, (unsigned)n), kRmsThreads, 0, stream>>>(static_cast<G *>(dgain), sums, cols, (int)ch.count, grad_stride, first);
        });
    });
    return launched(what);
}

int comp_ams_linear_q8_work_bytes(int64_t rows, int64_t cols, int64_t outs, int32_t q_aligned, int32_t w_aligned, uint64_t *bytes)
{
    const char *what = "linear_q8_work_bytes";
    if (const int rc = product_check(what, rows, cols, outs)) return rc;
    REQUIRE(bytes, "%s: bytes is NULL", what);
    *bytes = product_shape(rows, cols, outs, q_aligned != 0, w_aligned != 0).bytes;
    return COMP_AMS_OK;
}

int comp_ams_linear_q8(void *y, const int8_t *q, const float *scale, const int8_t *w, const float *w_scale, const float *bias,
                       int64_t rows, int64_t cols, int64_t outs, int64_t y_stride, int64_t q_stride, int64_t w_stride, int32_t type,
                       void *work, uint64_t work_bytes, void *hip_stream)
{
    const char *what = "linear_q8";
    REQUIRE(known_type(type), "%s: unknown type %d", what, type);
    if (const int rc = product_check(what, rows, cols, outs)) return rc;
    REQUIRE_BYTE_ROWS(what, "q", q, rows, cols, q_stride);
    REQUIRE_BYTE_ROWS(what, "w", w, outs, cols, w_stride);
    REQUIRE_ROWS(what, "y", y, outs ? rows : 0, outs, y_stride, type);
    REQUIRE((scale || rows == 0) && (w_scale || outs == 0), "%s: a scale is NULL", what);
    REQUIRE(aligned(scale, 4) && aligned(w_scale, 4) && aligned(bias, 4), "%s: scales and bias must be 4-byte aligned", what);
    // memory to LDS without registers: whole 16-byte chunks, and a tile's rows within 31 bits
    const bool q_aligned = cols % 16 == 0 && aligned(q, 16) && (rows <= 1 || (q_stride % 16 == 0 && q_stride < kMostStride));
    const bool w_aligned = cols % 16 == 0 && aligned(w, 16) && (outs <= 1 || (w_stride % 16 == 0 && w_stride < kMostStride));
    const ProductShape s = product_shape(rows, cols, outs, q_aligned, w_aligned);
    REQUIRE(s.bytes == 0 || (work && work_bytes >= s.bytes && aligned(work, 16)), "%s: needs %llu bytes of 16-byte aligned work memory", what,
            (unsigned long long)s.bytes);
    if (rows == 0 || outs == 0) return COMP_AMS_OK;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    ProductArgs a = {rows, outs, q_stride, w_stride, y_stride, (int)cols, (int)s.tiles_m, (int)s.tiles_n, s.splits, s.k_split, 0,
                     streamed_result(y, rows * outs, y_stride, 0, type)};
    const int64_t blocks = s.tiles_m * s.tiles_n * s.splits;
    int8_t *memory = static_cast<int8_t *>(work);
    if (!s.few && cols && !(q_aligned && w_aligned)) {
        PackArgs pa = {rows, outs, q_stride, w_stride, s.ld, (int)cols, shared_lanes(s.ld / 16), 0, 0};
        const int64_t blocks_x = q_aligned ? 0 : ceil_div(rows, kPackThreads / pa.lanes), blocks_w = w_aligned ? 0 : ceil_div(outs, kPackThreads / pa.lanes);
        REQUIRE(blocks_x + blocks_w <= kMaxBlocks, "%s: rows and outs are too many for one call", what);
        pa.blocks_x = (unsigned)blocks_x;
        in_launches(blocks_x + blocks_w, kPackThreads, [&](unsigned first, unsigned count) {
            pa.first = first;
            product8_pack<<<count, kPackThreads, 0, stream>>>(memory + s.x_at, memory + s.w_at, q, w, pa);
        });
        if (const int rc = launched(what)) return rc;          // what the product would read has not been written
        if (!q_aligned) q = memory + s.x_at, a.x_stride = s.ld;
        if (!w_aligned) w = memory + s.w_at, a.w_stride = s.ld;
        a.cols = (int)s.ld;
    }
    int *sums = reinterpret_cast<int *>(memory + s.sums_at);
    int rc = COMP_AMS_OK;
    with_type(type, [&](auto t) {
        using Y = decltype(t);
        Y *yt = static_cast<Y *>(y);
        if (s.few) {
            auto go = [&](auto kernel) {
                in_launches(blocks, kFewWaves * kWave, [&](unsigned first, unsigned count) {
                    a.first = first;
                    kernel<<<count, kFewWaves * kWave, 0, stream>>>(yt, q, scale, w, w_scale, bias, a);
                });
            };
            if (s.few == 1) go(product8_few<Y, 1>);
            else go(product8_few<Y, 2>);
            return;
        }
        auto go = [&](auto kernel, int threads) {
            in_launches(blocks, threads, [&](unsigned first, unsigned count) {
                a.first = first;
                kernel<<<count, threads, 0, stream>>>(yt, sums, q, scale, w, w_scale, bias, a);
            });
        };
        if (s.splits > 1) {
            if (s.high == 128) go(product8<Y, 128, 128, 2, 2, true>, 256);
            else go(product8<Y, 64, 64, 2, 2, true>, 256);
            rc = launched(what);                               // unless it is good, what the join would read has not been written
            if (rc) return;
            in_launches(ceil_div(ceil_div(outs, 4) * rows, kProductThreads), kProductThreads, [&](unsigned first, unsigned count) {
                a.first = first;
                product8_join<Y><<<count, kProductThreads, 0, stream>>>(yt, sums, scale, w_scale, bias, a);
            });
        } else if (s.high == 256) {
            if (s.wide == 256) go(product8<Y, 256, 256, 2, 4, false>, 512);
            else go(product8<Y, 256, 128, 4, 2, false>, 512);
        } else if (s.high == 128) {
            go(product8<Y, 128, 128, 2, 2, false>, 256);
        } else if (s.wide == 128) {
            go(product8<Y, 64, 128, 2, 2, false>, 256);
        } else {
            go(product8<Y, 64, 64, 2, 2, false>, 256);
        }
    });
    return rc ? rc : launched(what);
}

int comp_ams_linear_weight_grad_work_bytes(int64_t rows, int64_t cols, int64_t outs, int32_t n, int32_t binary, int32_t type, int32_t dy_aligned,
                                           uint64_t *bytes)
{
    const char *what = "linear_weight_grad_work_bytes";
    if (const int rc = weight_check(what, rows, cols, outs, n, binary, type)) return rc;
    REQUIRE(bytes, "%s: bytes is NULL", what);
    // for gradients of either width; and without a promise dy may be aligned all the same, where planes of q may take more than a copy of dy
    *bytes = 0;
    for (bool wide : {false, true})
        for (bool lies : {true, dy_aligned != 0}) *bytes = std::max(*bytes, weight_shape(rows, cols, outs, n, binary != 0, type, lies, wide).bytes);
    return COMP_AMS_OK;
}

int comp_ams_linear_weight_grad(void *dweight, void *dbias, const void *dy, const int8_t *q, const float *scale, int64_t rows,
                                int64_t cols, int64_t outs, int64_t dy_stride, int64_t q_stride, int32_t n, int64_t grad_stride,
                                int32_t in_first, int32_t binary, int32_t type, int32_t grad_type, void *work, uint64_t work_bytes,
                                void *hip_stream)
{
    const char *what = "linear_weight_grad";
    if (const int rc = weight_check(what, rows, cols, outs, n, binary, type)) return rc;
    REQUIRE(known_type(grad_type), "%s: unknown gradient type %d", what, grad_type);
    REQUIRE_BYTE_ROWS(what, "q", q, rows, cols, q_stride);
    REQUIRE_ROWS(what, "dy", dy, outs ? rows : 0, outs, dy_stride, type);
    REQUIRE_ROWS(what, "dweight", dweight, cols && outs ? (int64_t)n : 0, cols * outs, grad_stride, grad_type);
    if (dbias) REQUIRE_ROWS(what, "dbias", dbias, (int64_t)n, outs, grad_stride, grad_type);
    REQUIRE(scale || rows == 0, "%s: scale is NULL", what);
    REQUIRE(aligned(scale, 4), "%s: scale must be 4-byte aligned", what);
    if (rows <= 1) dy_stride = outs;       // any is allowed there, and the product takes the end of dy from it
    const bool dy_aligned = aligned(dy, 16) && dy_stride % 8 == 0 && dy_stride <= kMostChannels;
    const WeightShape s = weight_shape(rows, cols, outs, n, binary != 0, type, dy_aligned, grad_type == COMP_AMS_F32);
    REQUIRE(s.bytes == 0 || (work && work_bytes >= s.bytes && aligned(work, 16)), "%s: needs %llu bytes of 16-byte aligned work memory", what,
            (unsigned long long)s.bytes);
    if (outs == 0) return COMP_AMS_OK;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    char *memory = static_cast<char *>(work);
    float *sums = reinterpret_cast<float *>(memory + s.sums_at), *bias_sums = reinterpret_cast<float *>(memory + s.bias_at);
    const int64_t cells = cols * outs;
    if (cells == 0 && !dbias) return COMP_AMS_OK;
    weight_prepare_launch(s, memory, dy, q, scale, rows, cols, outs, dy_stride, q_stride, n, binary != 0, dbias != nullptr, type, stream);
    if (const int rc = launched(what)) return rc;              // what the product would read has not been written
    WeightArgs a = {};
    a.cols = cols, a.outs = outs, a.a_ld = s.a_ld, a.b_ld = s.copied ? s.b_ld : dy_stride;
    a.a_plane = s.q_planes > 1 ? rows * s.a_ld : 0, a.b_plane = s.dy_planes > 1 ? rows * s.b_ld : 0;
    a.worker_rows = rows / n, a.out_stride = in_first ? outs : cols;
    a.tiles_i = (int)s.tiles_i, a.tiles_o = (int)s.tiles_o, a.n = n, a.planes = s.q_planes * s.dy_planes;
    a.splits = (int)s.splits, a.split_steps = (int)s.split_steps;
    a.bias_chunks = (unsigned)s.bias_chunks, a.grad_stride = grad_stride;
    a.stream_out = s.splits == 1 && streamed_result(dweight, cells * n, a.out_stride, n > 1 ? grad_stride : 0, grad_type);
    const bf16_t *a_rows = reinterpret_cast<const bf16_t *>(memory + s.a_at);
    const bf16_t *b_rows = s.copied ? reinterpret_cast<const bf16_t *>(memory + s.b_at) : static_cast<const bf16_t *>(dy);
    if (s.splits > 1) {
        a.worker_stride = cells, a.piece_stride = cells * n;
        weight_launch<float>(sums, nullptr, a_rows, b_rows, nullptr, a, s.tile, in_first != 0, stream);
        if (const int rc = launched(what)) return rc;          // what the join would read has not been written
    } else {
        a.worker_stride = grad_stride;
    }
    with_type(grad_type, [&](auto t) {
        using G = decltype(t);
        if (s.splits == 1) {
            weight_launch<G>(static_cast<G *>(dweight), static_cast<G *>(dbias), a_rows, b_rows, bias_sums, a, s.tile, in_first != 0, stream);
            return;
        }
        const int64_t blocks = ceil_div(cells, 4 * kWeightJoinThreads);
        a.tiles = (unsigned)blocks;
        in_launches(blocks + (dbias ? ceil_div(outs, kWeightJoinThreads) : 0), kWeightJoinThreads, [&](unsigned first, unsigned count) {
            a.first = first;
            weight_join<G><<<dim3(count, (unsigned)n), kWeightJoinThreads, 0, stream>>>(static_cast<G *>(dweight), static_cast<G *>(dbias), sums, bias_sums,
                                                                                      cells, (int)s.splits, cells * n, a);
        });
    });
    return launched(what);
}

}  // extern "C"
