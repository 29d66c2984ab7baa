// Host side of include/comp_ams_operators.h: argument validation, the choice of kernels, launches.
#include "../../../include/comp_ams_operators.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "bias_kernels.h"
#include "norm_kernels.h"
#include "vocab_kernels.h"

using namespace cams_ops;

namespace {

thread_local char g_error[512] = "";

int fail(int code, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_error, sizeof g_error, fmt, ap);
    va_end(ap);
    return code;
}

// The status of the launches since the runtime's "last error" was clear; it is cleared again, or the caller's next HIP call
// would trip over it.
int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(COMP_AMS_EDEVICE, "%s: launch failed: %s", what, hipGetErrorString(e));
    return COMP_AMS_OK;
}

constexpr int64_t kMaxBlocks = ((int64_t)1 << 31) - 1;     // workgroups of a call, counted in 32 bits

// Workgroups of one launch: HIP takes fewer than 2^32 threads.
constexpr int64_t most_blocks(int threads) { return (((int64_t)1 << 32) - 1) / threads; }

// launch(first, count) for the workgroups [first, first + count) of a call, which has up to kMaxBlocks of them: one launch unless they are
// millions.
template <typename F>
void in_launches(int64_t blocks, int threads, F &&launch)
{
    const int64_t most = most_blocks(threads);
    for (int64_t first = 0; first < blocks; first += most) launch((unsigned)first, (unsigned)std::min(blocks - first, most));
}
constexpr int64_t kMaxElements = (int64_t)1 << 60;    // rows * stride: offsets in bytes stay far below 2^63

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

size_t type_size(int32_t type) { return type == COMP_AMS_F32 ? 4 : 2; }
bool known_type(int32_t type) { return type == COMP_AMS_F32 || type == COMP_AMS_BF16 || type == COMP_AMS_F16; }
bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Calls f with a value of the element type.
template <typename F>
void with_type(int32_t type, F &&f)
{
    if (type == COMP_AMS_F32) f(float{});
    else if (type == COMP_AMS_BF16) f(bf16_t{});
    else f(f16_t{});
}

#define REQUIRE(cond, ...)                                        \
    do {                                                          \
        if (!(cond)) return fail(COMP_AMS_EINVAL, __VA_ARGS__);   \
    } while (0)

// A strided array of rows: base pointer, alignment, stride of at least a row, offsets in range.
#define REQUIRE_ROWS(what, name, p, rows, cols, stride, type)                                                                  \
    do {                                                                                                                       \
        REQUIRE((p) != nullptr || (rows) == 0, "%s: %s is NULL", what, name);                                                  \
        REQUIRE(aligned(p, type_size(type)), "%s: %s must be %zu-byte aligned", what, name, type_size(type));                   \
        REQUIRE((stride) >= (cols) || (rows) <= 1, "%s: the rows of %s overlap (stride %lld < %lld)", what, name,              \
                (long long)(stride), (long long)(cols));                                                                       \
        REQUIRE((stride) >= 0 && ((rows) <= 1 || (stride) < kMaxElements / (rows)), "%s: %s is out of range", what, name);        \
    } while (0)

// Whether an array that a call reads or writes once is streamed past the caches.  What is written is read by the model's next
// operation, if anything of it is left in the 256 MB memory-side cache by then; what is read was written by the one before.
bool streamed_out(int64_t elements, int32_t type) { return elements > ((int64_t)80 << 20) / (int64_t)type_size(type); }
bool streamed_in(int64_t elements, int32_t type) { return elements > ((int64_t)256 << 20) / (int64_t)type_size(type); }

// --- constants chosen from sizes, as types ---------------------------------------------------------------------------

// f(Shape) with `vecs`, in [kLeast, kVecs], as a compile-time constant: a row of more than (vecs - 1) kThreads vectors.
// sure: slabs that are known to be full.
template <int kThreads, int kVecs, int kSure = (kVecs > 0 ? kVecs - 1 : 0)> struct Shape {
    static constexpr int threads = kThreads, vecs = kVecs, sure = kSure;
};
template <int kThreads, int kLeast, int kVecs, typename F>
void with_vecs(int vecs, F &&f)
{
    if constexpr (kVecs == kLeast) {
        f(Shape<kThreads, kVecs>{});
    } else {
        if (vecs >= kVecs) f(Shape<kThreads, kVecs>{});
        else with_vecs<kThreads, kLeast, kVecs - 1>(vecs, f);
    }
}

// f(Shape) with the team of lanes and the vectors a lane that hold a row of `len` elements in registers: 16 lanes up to 32 vectors,
// a wavefront up to 256, a workgroup of 256 up to 1024, of 1024 up to 2048.  false if the row is longer than that, or shorter than a
// vector.
template <typename T, typename F>
bool with_team(int64_t len, F &&f)
{
    const int64_t vecs = ceil_div(len, kVec<T>);
    if (len < kVec<T>) return false;
    if (vecs <= 32) with_vecs<16, 1, 2>((int)ceil_div(vecs, 16), f);
    else if (vecs <= 256) with_vecs<64, 1, 4>((int)ceil_div(vecs, 64), f);
    else if (vecs <= 1024) with_vecs<256, 2, 4>((int)ceil_div(vecs, 256), f);
    else if (vecs <= 2048) f(Shape<1024, 2>{});
    else return false;
    return true;
}

// --- layer norm ---------------------------------------------------------------------------------------------------

int norm_check(const char *what, int64_t rows, int64_t cols, int32_t type)
{
    REQUIRE(known_type(type), "%s: unknown type %d", what, type);
    REQUIRE(rows >= 0 && rows < (int64_t)1 << 40, "%s: rows=%lld must be in [0, 2^40)", what, (long long)rows);
    REQUIRE(cols >= 1 && cols < (int64_t)1 << 31, "%s: cols=%lld must be in [1, 2^31)", what, (long long)cols);
    return COMP_AMS_OK;
}

// Workgroups of the forward pass: enough to fill the chip, few enough that a team keeps gain and shift in registers over several rows.
// 16384 x 768 bf16, us: 1024 13.4, 2048 13.5, 4096 and 8192 (a row a team) 18.
constexpr int64_t kNormBlocks = 2048;
// Workgroups that the rows of all workers are cut into in the backward pass.  More keep more rows in flight, and write more partial
// sums.  us at 512 / 768 / 1024 / 1280: 16384 x 768 bf16, n = 8 20.7 / 21.3 / 19.6 / 19.7; 20000 x 2047 fp32, n = 20 125 / 118 / 115 / 121.
constexpr int64_t kNormChunkBlocks = 1024;

// How a worker's rows are cut for the parameter gradients: chunks of rows with one set of column sums each.
struct NormChunks {
    int64_t rows, count;     // rows of a chunk; chunks of a worker
};
NormChunks norm_chunks(int64_t worker_rows, int32_t n)
{
    const int64_t want = std::max<int64_t>(1, ceil_div(kNormChunkBlocks, n));
    const int64_t rows = std::max<int64_t>(16, ceil_div(worker_rows, want));
    return {rows, std::max<int64_t>(1, ceil_div(worker_rows, rows))};
}

// --- the biased softmax ---------------------------------------------------------------------------------------------

int bias_check(const char *what, const int32_t *bounds, int32_t n_buckets, const int32_t *key_len, int64_t batch, int64_t heads,
               int64_t tq, int64_t tk, int64_t offset, float scale, int32_t type, Bounds *out)
{
    REQUIRE(known_type(type), "%s: unknown type %d", what, type);
    REQUIRE(n_buckets >= 1 && n_buckets <= COMP_AMS_MAX_BUCKETS, "%s: n_buckets=%d must be in [1, %d]", what, n_buckets,
            COMP_AMS_MAX_BUCKETS);
    REQUIRE(bounds || n_buckets == 1, "%s: bounds are NULL", what);
    REQUIRE(batch >= 0 && heads >= 0 && tq >= 0 && tk >= 0, "%s: a size is negative", what);
    REQUIRE(tk < (int64_t)1 << 31, "%s: tk=%lld must be below 2^31", what, (long long)tk);
    const int64_t most = (int64_t)1 << 31;
    REQUIRE(batch < most && heads < most && tq < most / 2, "%s: a size is out of range", what);
    if (batch && heads && tq)
        REQUIRE(batch * heads < most && batch * heads * tq < most, "%s: batch*heads*tq must be below 2^31", what);
    REQUIRE(offset > -most && offset < most, "%s: offset out of range", what);
    REQUIRE(std::isfinite(scale), "%s: scale must be finite", what);
    REQUIRE(aligned(key_len, 4), "%s: key_len must be 4-byte aligned", what);
    out->n = n_buckets - 1;
    for (int32_t q = 0; q < n_buckets - 1; ++q) {
        REQUIRE(q == 0 || bounds[q] > bounds[q - 1], "%s: bounds must be strictly ascending (bound %d)", what, q);
        out->at[q] = bounds[q];
    }
    return COMP_AMS_OK;
}

// One array of [batch][heads][tq] rows.
int bias_strides(const char *what, const char *name, const void *p, int64_t batch, int64_t heads, int64_t tq, int64_t tk,
                 const int64_t *st, int32_t type)
{
    REQUIRE(p, "%s: %s is NULL", what, name);
    REQUIRE(aligned(p, type_size(type)), "%s: %s must be %zu-byte aligned", what, name, type_size(type));
    const int64_t size[3] = {batch, heads, tq};
    for (int q = 0; q < 3; ++q) {
        if (size[q] <= 1) continue;
        REQUIRE(st[q] >= tk, "%s: the rows of %s overlap (stride %lld < %lld)", what, name, (long long)st[q], (long long)tk);
        REQUIRE(st[q] < kMaxElements / size[q], "%s: %s is out of range", what, name);
    }
    return COMP_AMS_OK;
}

// Workgroups of the forward pass, each with its own layout of a head's bias in LDS: more of them hide each other's latency, fewer lay out
// less.  us at 1536 / 2048 / 3072: wavefronts over many rows 16 x 12 x 512 x 512 bf16 44 / 41 / 40, 8 x 12 x 1024 x 1024 100 / 100 / 90;
// over few 8 x 8 x 300 x 300 12.3 / 12.3 / 13.6; teams of 16 lanes 64 x 8 x 128 x 128 10.0 / 11.1 / 11.3; workgroups 2 x 16 x 2000 x 2000
// f16 120 / 144 / 126.
int64_t bias_forward_blocks(int team, int64_t rows) { return team == 64 && rows >= 65536 ? 3072 : 1536; }

// How the queries of a head and sequence are cut for the backward pass: the registers' form takes rows_team consecutive queries a team.
struct BiasShape {
    bool held;               // false: bias_backward_any
    int32_t team, rows_team, rows_block;
    int64_t pieces;
};
// A wavefront takes a row of up to 128 vectors, a workgroup longer ones: by the wavefront, four teams' arrays over the positions leave room
// for three workgroups a compute unit (2 x 16 x 1999 x 1999 f16 causal: 194 us against 136).
// The rows a team takes: as many as leave kBiasBackwardBlocks workgroups, between a step's and 32.  us at 16 x 12 x 512 x 512 bf16 / the
// causal case: at least 640 workgroups 59 / 136, 1600 53 / 136, 3200 49 / 121, 6400 47 / 113.
constexpr int64_t kBiasBackwardBlocks = 6400;
BiasShape bias_backward_shape(int64_t sequences, int64_t tq, int64_t tk, int32_t type)
{
    const int64_t e = 16 / (int64_t)type_size(type), vecs = ceil_div(std::max<int64_t>(tk, 1), e);
    if (tk < e || vecs > 1024) return {false, 0, kBiasAnyRows, kBiasAnyRows, ceil_div(tq, kBiasAnyRows)};
    const int32_t team = vecs <= 32 ? 16 : vecs <= 128 ? 64 : 256, teams = kTeamBlock<256> / team;
    int32_t rows = 32;
    while (rows > e && sequences * ceil_div(tq, rows * teams) < kBiasBackwardBlocks) rows /= 2;
    return {true, team, rows, rows * teams, ceil_div(tq, rows * teams)};
}

// --- vocabulary rows ----------------------------------------------------------------------------------------------------

int vocab_sizes(const char *what, int64_t rows, int64_t vocab, int32_t type)
{
    REQUIRE(known_type(type), "%s: unknown type %d", what, type);
    REQUIRE(rows >= 0 && rows < (int64_t)1 << 31, "%s: rows=%lld must be in [0, 2^31)", what, (long long)rows);
    REQUIRE(vocab >= 1 && vocab < (int64_t)1 << 31, "%s: vocab=%lld must be in [1, 2^31)", what, (long long)vocab);
    return COMP_AMS_OK;
}

int vocab_check(const char *what, const void *logits, int64_t rows, int64_t vocab, int64_t stride, int32_t type)
{
    if (const int rc = vocab_sizes(what, rows, vocab, type)) return rc;
    REQUIRE_ROWS(what, "logits", logits, rows, vocab, stride, type);
    return COMP_AMS_OK;
}

int distill_check(const char *what, const void *logits, const int32_t *idx, const float *val, int64_t rows, int64_t vocab,
                  int64_t stride, int32_t k, float temperature, int32_t type)
{
    if (const int rc = vocab_check(what, logits, rows, vocab, stride, type)) return rc;
    REQUIRE(k >= 1 && k <= COMP_AMS_MAX_TOP, "%s: k=%d must be in [1, %d]", what, k, COMP_AMS_MAX_TOP);
    REQUIRE(std::isfinite(temperature) && temperature > 0.f && std::isfinite(1.f / temperature * kLog2e),
            "%s: temperature must be positive and finite, and so must its reciprocal in units of log 2", what);
    REQUIRE((idx && val) || rows == 0, "%s: idx or val is NULL", what);
    REQUIRE(aligned(idx, 4) && aligned(val, 4), "%s: idx and val must be 4-byte aligned", what);
    return COMP_AMS_OK;
}

// How a row of a vocabulary is cut for logprobs_regs, and which of its forms takes a piece.
struct PieceShape {
    int32_t count;           // pieces of a row; 0: the row is too long, or shorter than a vector: logprobs_any
    int64_t len;             // elements of a piece, a multiple of 64 unless there is one only
    int32_t threads, vecs;
};

PieceShape piece_shape(int64_t rows, int64_t vocab, int32_t type)
{
    const int64_t lanes = (int64_t)kPieceThreads * 16 / (int64_t)type_size(type);     // elements of one vector of every thread
    PieceShape s = {1, vocab, kPieceThreads, 1};
    if (vocab < 16 / (int64_t)type_size(type)) return {0, 0, 0, 0};
    if (vocab <= lanes / 2) {
        s.threads = kPieceThreads / 2;
        return s;
    }
    const int64_t count = ceil_div(vocab, lanes * kPieceVecs);
    if (count > kMaxPieces || rows * count > kMaxBlocks) return {0, 0, 0, 0};
    s.count = (int32_t)count;
    if (count > 1) s.len = ceil_div(ceil_div(vocab, count), 64) * 64;
    s.vecs = (int32_t)ceil_div(s.len, lanes);
    return s;
}

}  // namespace

extern "C" {

const char *comp_ams_operators_last_error(void) { return g_error; }

int comp_ams_layer_norm(void *y, float *mean, float *rstd, const void *x, const float *gain, const float *shift, int64_t rows,
                        int64_t cols, int64_t x_stride, int64_t y_stride, float eps, int32_t type, void *hip_stream)
{
    const char *what = "layer_norm";
    if (const int rc = norm_check(what, rows, cols, type)) return rc;
    REQUIRE_ROWS(what, "x", x, rows, cols, x_stride, type);
    REQUIRE_ROWS(what, "y", y, rows, cols, y_stride, type);
    REQUIRE(gain, "%s: gain is NULL", what);
    REQUIRE(aligned(gain, 4) && aligned(shift, 4) && aligned(mean, 4) && aligned(rstd, 4), "%s: gain, shift, mean and rstd must be 4-byte aligned", what);
    REQUIRE(std::isfinite(eps) && eps >= 0.f, "%s: eps must be finite and not negative", what);
    if (rows == 0) return COMP_AMS_OK;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const NormArgs a = {rows, cols, x_stride, y_stride, 0, eps, (float)(1.0 / (double)cols), streamed_out(rows * cols, type)};
    with_type(type, [&](auto t) {
        using T = decltype(t);
        const bool held = with_team<T>(cols, [&](auto shape) {
            using S = decltype(shape);
            const int64_t teams = kTeamBlock<S::threads> / S::threads;
            norm_forward<T, S::threads, S::vecs><<<(unsigned)std::min<int64_t>(ceil_div(rows, teams), kNormBlocks), kTeamBlock<S::threads>, 0, stream>>>(
                static_cast<T *>(y), mean, rstd, static_cast<const T *>(x), gain, shift, a);
        });
        if (!held)
            norm_forward_any<T><<<(unsigned)std::min(rows, most_blocks(kNormThreads)), kNormThreads, 0, stream>>>(static_cast<T *>(y), mean, rstd,
                                                                                              static_cast<const T *>(x), gain, shift, a);
    });
    return launched(what);
}

int comp_ams_layer_norm_work_bytes(int64_t rows, int64_t cols, int32_t n, uint64_t *bytes)
{
    const char *what = "layer_norm_work_bytes";
    if (const int rc = norm_check(what, rows, cols, COMP_AMS_F32)) return rc;
    REQUIRE(n >= 1 && n <= 65535, "%s: n=%d must be in [1, 65535]", what, n);
    REQUIRE(rows % n == 0, "%s: rows=%lld must be a multiple of n=%d", what, (long long)rows, n);
    REQUIRE(bytes, "%s: bytes is NULL", what);
    *bytes = (uint64_t)norm_chunks(rows / n, n).count * (uint64_t)n * 2u * (uint64_t)cols * sizeof(float);
    return COMP_AMS_OK;
}

int comp_ams_layer_norm_backward(void *dx, void *dgain, void *dshift, const void *dy, const void *x, const float *mean,
                                 const float *rstd, const float *gain, int64_t rows, int64_t cols, int64_t dx_stride, int64_t dy_stride,
                                 int64_t x_stride, int32_t n, int64_t grad_stride, int32_t type, int32_t grad_type, void *work,
                                 uint64_t work_bytes, void *hip_stream)
{
    const char *what = "layer_norm_backward";
    if (const int rc = norm_check(what, rows, cols, type)) return rc;
    REQUIRE(known_type(grad_type), "%s: unknown gradient type %d", what, grad_type);
    REQUIRE(n >= 1 && n <= 65535, "%s: n=%d must be in [1, 65535]", what, n);
    REQUIRE(rows % n == 0, "%s: rows=%lld must be a multiple of n=%d", what, (long long)rows, n);
    REQUIRE_ROWS(what, "x", x, rows, cols, x_stride, type);
    REQUIRE_ROWS(what, "dy", dy, rows, cols, dy_stride, type);
    REQUIRE_ROWS(what, "dx", dx, rows, cols, dx_stride, type);
    REQUIRE_ROWS(what, "dgain", dgain, (int64_t)n, cols, grad_stride, grad_type);
    REQUIRE(aligned(dshift, type_size(grad_type)), "%s: dshift must be %zu-byte aligned", what, type_size(grad_type));
    REQUIRE(gain && ((mean && rstd) || rows == 0), "%s: mean, rstd or gain is NULL", what);
    REQUIRE(aligned(gain, 4) && aligned(mean, 4) && aligned(rstd, 4), "%s: mean, rstd and gain must be 4-byte aligned", what);
    uint64_t need = 0;
    if (const int rc = comp_ams_layer_norm_work_bytes(rows, cols, n, &need)) return rc;
    REQUIRE(work && work_bytes >= need, "%s: needs %llu bytes of work memory", what, (unsigned long long)need);
    REQUIRE(aligned(work, 16), "%s: work must be 16-byte aligned", what);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const NormArgs a = {rows, cols, x_stride, dx_stride, dy_stride, 0.f, (float)(1.0 / (double)cols), streamed_out(rows * cols, type)};
    const NormChunks ch = norm_chunks(rows / n, n);
    float *sums = static_cast<float *>(work);
    with_type(type, [&](auto t) {
        using T = decltype(t);
        const bool held = with_team<T>(cols, [&](auto shape) {
            using S = decltype(shape);
            norm_backward<T, S::threads, S::vecs><<<dim3((unsigned)ch.count, (unsigned)n), kTeamBlock<S::threads>, 0, stream>>>(
                static_cast<T *>(dx), sums, static_cast<const T *>(dy), static_cast<const T *>(x), mean, rstd, gain, a, rows / n, ch.rows);
        });
        if (held) return;
        // the parameter gradients first: dx may replace dy or x
        norm_param_any<T><<<dim3((unsigned)ceil_div(cols, kNormThreads), (unsigned)ch.count, (unsigned)n), kNormThreads, 0, stream>>>(
            sums, static_cast<const T *>(dy), static_cast<const T *>(x), mean, rstd, a, rows / n, ch.rows);
        if (rows > 0)
            norm_backward_any<T><<<(unsigned)std::min(rows, most_blocks(kNormThreads)), kNormThreads, 0, stream>>>(
                static_cast<T *>(dx), static_cast<const T *>(dy), static_cast<const T *>(x), mean, rstd, gain, a);
    });
    if (const int rc = launched(what)) return rc;              // what the join would read has not been written
    with_type(grad_type, [&](auto t) {
        using G = decltype(t);
        in_launches(ceil_div(2 * cols, kJoinCols), kNormThreads, [&](unsigned first, unsigned count) {
            norm_param_join<G><<<dim3(count, (unsigned)n), kNormThreads, 0, stream>>>(static_cast<G *>(dgain), static_cast<G *>(dshift), sums,
                                                                                    cols, (int)ch.count, grad_stride, first);
        });
    });
    return launched(what);
}

int comp_ams_rel_bias_softmax(void *p, const void *s, const float *table, const int32_t *bounds_host, int32_t n_buckets,
                              const int32_t *key_len, int64_t batch, int64_t heads, int64_t tq, int64_t tk,
                              const int64_t *p_strides_host, const int64_t *s_strides_host, int64_t offset, float scale,
                              int32_t causal, int32_t type, void *hip_stream)
{
    const char *what = "rel_bias_softmax";
    Bounds bounds;
    if (const int rc = bias_check(what, bounds_host, n_buckets, key_len, batch, heads, tq, tk, offset, scale, type, &bounds)) return rc;
    if (batch == 0 || heads == 0 || tq == 0 || tk == 0) return COMP_AMS_OK;
    REQUIRE(p_strides_host && s_strides_host, "%s: strides are NULL", what);
    if (const int rc = bias_strides(what, "p", p, batch, heads, tq, tk, p_strides_host, type)) return rc;
    if (const int rc = bias_strides(what, "s", s, batch, heads, tq, tk, s_strides_host, type)) return rc;
    REQUIRE(table && aligned(table, 4), "%s: table is NULL or not 4-byte aligned", what);
    BiasArgs a = {};
    a.heads = heads, a.tq = tq, a.tk = tk, a.rows = batch * heads * tq;
    a.s_b = s_strides_host[0], a.s_h = s_strides_host[1], a.s_q = s_strides_host[2];
    a.p_b = p_strides_host[0], a.p_h = p_strides_host[1], a.p_q = p_strides_host[2];
    a.offset = offset, a.scale = scale, a.causal = causal != 0, a.stream_out = streamed_out(a.rows * tk, type);
    with_type(type, [&](auto t) {
        using T = decltype(t);
        const int64_t vecs = ceil_div(tk, kVec<T>);
        auto launch = [&](auto shape) {
            using S = decltype(shape);
            constexpr int kTeams = kTeamBlock<S::threads> / S::threads;
            const int64_t share = std::max<int64_t>(1, ceil_div(a.rows, bias_forward_blocks(S::threads, a.rows) * kTeams)) * kTeams;
            const int rows_block = (int)std::min<int64_t>(tq, std::min<int64_t>(256, share));
            const int64_t pieces = ceil_div(tq, rows_block);
            const size_t lds = (size_t)(tk + rows_block - 1) * sizeof(float);
            in_launches(batch * heads * pieces, kTeamBlock<S::threads>, [&](unsigned first, unsigned count) {
                a.first = first;
                bias_forward<T, S::threads, S::vecs><<<count, kTeamBlock<S::threads>, lds, static_cast<hipStream_t>(hip_stream)>>>(
                    static_cast<T *>(p), static_cast<const T *>(s), table, bounds, key_len, a, (int)pieces, rows_block);
            });
        };
        // rows of more than 128 vectors by a workgroup: by a wavefront they take 150 registers (2 x 16 x 2000 x 2000 f16 172 us against 119)
        if (tk >= kVec<T> && vecs <= 1024) {
            if (vecs <= 32) with_vecs<16, 1, 2>((int)ceil_div(vecs, 16), launch);
            else if (vecs <= 128) with_vecs<64, 1, 2>((int)ceil_div(vecs, 64), launch);
            else with_vecs<256, 1, 4>((int)ceil_div(vecs, 256), launch);
            return;
        }
        bias_forward_any<T><<<(unsigned)std::min(a.rows, most_blocks(kBiasThreads)), kBiasThreads, 0, static_cast<hipStream_t>(hip_stream)>>>(
            static_cast<T *>(p), static_cast<const T *>(s), table, bounds, key_len, a);
    });
    return launched(what);
}

int comp_ams_rel_bias_work_bytes(int64_t batch, int64_t heads, int64_t tq, int64_t tk, int32_t n_buckets, int32_t type, uint64_t *bytes)
{
    const char *what = "rel_bias_work_bytes";
    Bounds none;
    if (const int rc = bias_check(what, nullptr, 1, nullptr, batch, heads, tq, tk, 0, 1.f, type, &none)) return rc;
    REQUIRE(n_buckets >= 1 && n_buckets <= COMP_AMS_MAX_BUCKETS, "%s: n_buckets=%d must be in [1, %d]", what, n_buckets, COMP_AMS_MAX_BUCKETS);
    REQUIRE(bytes, "%s: bytes is NULL", what);
    *bytes = (uint64_t)(batch * heads * bias_backward_shape(batch * heads, tq, tk, type).pieces) * (uint64_t)n_buckets * sizeof(float);
    return COMP_AMS_OK;
}

int comp_ams_rel_bias_softmax_backward(void *ds, void *dtable, const void *dp, const void *p, const int32_t *bounds_host,
                                       int32_t n_buckets, const int32_t *key_len, int64_t batch, int64_t heads, int64_t tq,
                                       int64_t tk, const int64_t *strides_host, int64_t offset, float scale, int32_t causal,
                                       int32_t n, int64_t grad_stride, int32_t type, int32_t grad_type, void *work,
                                       uint64_t work_bytes, void *hip_stream)
{
    const char *what = "rel_bias_softmax_backward";
    Bounds bounds;
    if (const int rc = bias_check(what, bounds_host, n_buckets, key_len, batch, heads, tq, tk, offset, scale, type, &bounds)) return rc;
    REQUIRE(known_type(grad_type), "%s: unknown gradient type %d", what, grad_type);
    REQUIRE(n >= 1 && n <= 65535, "%s: n=%d must be in [1, 65535]", what, n);
    REQUIRE(batch % n == 0, "%s: batch=%lld must be a multiple of n=%d", what, (long long)batch, n);
    if (heads == 0) return COMP_AMS_OK;
    REQUIRE(heads <= 65535, "%s: heads=%lld must be at most 65535", what, (long long)heads);
    REQUIRE_ROWS(what, "dtable", dtable, (int64_t)n, (int64_t)n_buckets * heads, grad_stride, grad_type);
    const bool empty = batch == 0 || tq == 0 || tk == 0;
    uint64_t need = 0;
    if (!empty) {
        REQUIRE(strides_host, "%s: strides are NULL", what);
        if (const int rc = bias_strides(what, "ds", ds, batch, heads, tq, tk, strides_host, type)) return rc;
        if (const int rc = bias_strides(what, "dp", dp, batch, heads, tq, tk, strides_host + 3, type)) return rc;
        if (const int rc = bias_strides(what, "p", p, batch, heads, tq, tk, strides_host + 6, type)) return rc;
        if (const int rc = comp_ams_rel_bias_work_bytes(batch, heads, tq, tk, n_buckets, type, &need)) return rc;
        REQUIRE(work && work_bytes >= need, "%s: needs %llu bytes of work memory", what, (unsigned long long)need);
        REQUIRE(aligned(work, 16), "%s: work must be 16-byte aligned", what);
    }
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    float *sums = static_cast<float *>(work);
    const BiasShape cut = bias_backward_shape(batch * heads, tq, tk, type);
    if (!empty) {
        BiasArgs a = {};
        a.heads = heads, a.tq = tq, a.tk = tk, a.rows = batch * heads * tq;
        a.o_b = strides_host[0], a.o_h = strides_host[1], a.o_q = strides_host[2];
        a.s_b = strides_host[3], a.s_h = strides_host[4], a.s_q = strides_host[5];
        a.p_b = strides_host[6], a.p_h = strides_host[7], a.p_q = strides_host[8];
        a.offset = offset, a.scale = scale, a.causal = causal != 0, a.stream_out = streamed_out(a.rows * tk, type);
        with_type(type, [&](auto t) {
            using T = decltype(t);
            const int64_t blocks = batch * heads * cut.pieces;
            if (!cut.held) {
                in_launches(blocks, kBiasAnyThreads, [&](unsigned first, unsigned count) {
                    a.first = first;
                    bias_backward_any<T><<<count, kBiasAnyThreads, 0, stream>>>(static_cast<T *>(ds), sums, static_cast<const T *>(dp),
                                                                               static_cast<const T *>(p), bounds, key_len, a, cut.pieces, batch / n);
                });
                return;
            }
            auto launch = [&](auto shape) {
                using S = decltype(shape);
                // Longer rows one at a time (and one on its way), or the registers leave three wavefronts a SIMD: 64 x 8 x 250 x 250 f16 70 us
                // against 54, 2 x 16 x 1500 x 1500 fp32 194 against 172.  Single vectors by twos: the causal case 115 against 120.
                constexpr int kTeams = kTeamBlock<S::threads> / S::threads, kStep = 4, kBatch = S::vecs > 1 ? 1 : 2;
                constexpr int kSlots = S::threads * S::vecs * kVec<T>;
                const size_t lds = ((size_t)kTeams * (kSlots + cut.rows_team - 1) + (kTeams > 1 ? kSlots + cut.rows_block - 1 : 0)) * sizeof(float);
                in_launches(blocks, kTeamBlock<S::threads>, [&](unsigned first, unsigned count) {
                    a.first = first;
                    bias_backward<T, S::threads, S::vecs, kStep, kBatch><<<count, kTeamBlock<S::threads>, lds, stream>>>(
                        static_cast<T *>(ds), sums, static_cast<const T *>(dp), static_cast<const T *>(p), bounds, key_len, a,
                        (int)cut.pieces, cut.rows_team, (unsigned)(batch / n));
                });
            };
            const int vecs = (int)ceil_div(tk, kVec<T>);
            if (cut.team == 16) with_vecs<16, 1, 2>(ceil_div(vecs, 16), launch);
            else if (cut.team == 64) with_vecs<64, 1, 2>(ceil_div(vecs, 64), launch);
            else with_vecs<256, 1, 4>(ceil_div(vecs, 256), launch);
        });
        if (const int rc = launched(what)) return rc;          // what the join would read has not been written
    }
    with_type(grad_type, [&](auto t) {
        using G = decltype(t);
        bias_table_join<G><<<dim3((unsigned)n_buckets, (unsigned)heads, (unsigned)n), kWave, 0, stream>>>(
            static_cast<G *>(dtable), sums, heads, empty ? 0 : batch / n * cut.pieces, n_buckets, grad_stride);
    });
    return launched(what);
}

int comp_ams_token_logprobs_work_bytes(int64_t rows, int64_t vocab, int32_t k, int32_t type, uint64_t *bytes)
{
    const char *what = "token_logprobs_work_bytes";
    if (const int rc = vocab_sizes(what, rows, vocab, type)) return rc;
    REQUIRE(k >= 0 && k <= COMP_AMS_MAX_TOP && k <= vocab, "%s: k=%d must be in [0, min(vocab, %d)]", what, k, COMP_AMS_MAX_TOP);
    REQUIRE(bytes, "%s: bytes is NULL", what);
    const PieceShape s = piece_shape(rows, vocab, type);
    *bytes = s.count > 1 ? (uint64_t)rows * (uint64_t)s.count * ((uint64_t)k * sizeof(uint64_t) + sizeof(Piece)) : 0;
    return COMP_AMS_OK;
}

int comp_ams_token_logprobs(float *logp, float *entropy, int32_t *top_idx, float *top_logp, const void *logits, const int64_t *tokens,
                            int64_t rows, int64_t vocab, int64_t stride, int32_t k, int32_t type, void *work, uint64_t work_bytes,
                            void *hip_stream)
{
    const char *what = "token_logprobs";
    if (const int rc = vocab_check(what, logits, rows, vocab, stride, type)) return rc;
    REQUIRE(k >= 0 && k <= COMP_AMS_MAX_TOP && k <= vocab, "%s: k=%d must be in [0, min(vocab, %d)]", what, k, COMP_AMS_MAX_TOP);
    REQUIRE(k == 0 || (top_idx && top_logp) || rows == 0, "%s: top_idx or top_logp is NULL", what);
    REQUIRE(!logp || tokens, "%s: logp needs tokens", what);
    REQUIRE(aligned(logp, 4) && aligned(entropy, 4) && aligned(top_idx, 4) && aligned(top_logp, 4) && aligned(tokens, 8),
            "%s: an array is not aligned to its elements", what);
    uint64_t need = 0;
    if (const int rc = comp_ams_token_logprobs_work_bytes(rows, vocab, k, type, &need)) return rc;
    REQUIRE(need == 0 || (work && work_bytes >= need && aligned(work, 16)), "%s: needs %llu bytes of 16-byte aligned work memory", what,
            (unsigned long long)need);
    if (rows == 0) return COMP_AMS_OK;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const PieceShape s = piece_shape(rows, vocab, type);
    int rc = COMP_AMS_OK;
    with_type(type, [&](auto t) {
        using T = decltype(t);
        const T *z = static_cast<const T *>(logits);
        if (s.count == 0) {
            logprobs_any<T><<<(unsigned)std::min(rows, most_blocks(kVocabThreads)), kVocabThreads, 0, stream>>>(logp, entropy, top_idx, top_logp, z, tokens, rows, vocab, stride, k);
            return;
        }
        uint64_t *keys = static_cast<uint64_t *>(work);
        Piece *pieces = reinterpret_cast<Piece *>(keys + (s.count > 1 ? rows * s.count * k : 0));
        const int groups = k <= 32 ? 64 : k <= 64 ? 128 : 256;
        auto launch = [&](auto shape) {
            using S = decltype(shape);
            in_launches(rows * s.count, S::threads, [&](unsigned first, unsigned count) {
                logprobs_regs<T, S::threads, S::vecs><<<count, S::threads, 0, stream>>>(
                    logp, entropy, top_idx, top_logp, z, tokens, vocab, stride, k, groups, s.count, s.len,
                    s.len < (int64_t)S::threads * S::vecs * kVec<T> ? 1 : 0, pieces, keys, first);
            });
        };
        if (s.threads == kPieceThreads) with_vecs<kPieceThreads, 1, kPieceVecs>(s.vecs, launch);
        else launch(Shape<kPieceThreads / 2, 1>{});
        rc = launched(what);                                   // unless it is good, what the join would read has not been written
        if (rc == COMP_AMS_OK && s.count > 1)
            in_launches(rows, kVocabThreads, [&](unsigned first, unsigned count) {
                logprobs_join<T><<<count, kVocabThreads, (size_t)s.count * k * sizeof(uint64_t), stream>>>(
                    logp, entropy, top_idx, top_logp, z, tokens, vocab, stride, k, s.count, pieces, keys, first);
            });
    });
    return rc ? rc : launched(what);
}

int comp_ams_distill(float *loss, float *lse, const void *logits, const int32_t *idx, const float *val, int64_t rows, int64_t vocab,
                     int64_t stride, int32_t k, float temperature, int32_t type, void *hip_stream)
{
    const char *what = "distill";
    if (const int rc = distill_check(what, logits, idx, val, rows, vocab, stride, k, temperature, type)) return rc;
    REQUIRE(aligned(loss, 4) && aligned(lse, 4), "%s: loss and lse must be 4-byte aligned", what);
    if (rows == 0) return COMP_AMS_OK;
    DistillArgs a = {rows, vocab, stride, 0, k, temperature, 1.f / temperature, streamed_in(rows * vocab, type), streamed_out(rows * vocab, type), 0};
    with_type(type, [&](auto t) {
        using T = decltype(t);
        auto launch = [&](auto shape) {
            using S = decltype(shape);
            in_launches(rows, S::threads, [&](unsigned first, unsigned count) {
                a.first = first;
                distill_forward<T, S::threads><<<count, S::threads, 0, static_cast<hipStream_t>(hip_stream)>>>(
                    loss, lse, static_cast<const T *>(logits), idx, val, a);
            });
        };
        if (vocab < kVec<T>)
            in_launches(rows, kVocabThreads, [&](unsigned first, unsigned count) {
                a.first = first;
                distill_any<T, true, false><<<count, kVocabThreads, 0, static_cast<hipStream_t>(hip_stream)>>>(
                    loss, lse, nullptr, nullptr, static_cast<const T *>(logits), nullptr, idx, val, a);
            });
        else if (rows >= 1024 || vocab <= 4 * 256 * kVec<T>) launch(Shape<256, 0>{});
        else launch(Shape<1024, 0>{});
    });
    return launched(what);
}

int comp_ams_distill_backward(void *dlogits, const float *dloss, const void *logits, const float *lse, const int32_t *idx,
                              const float *val, int64_t rows, int64_t vocab, int64_t dlogits_stride, int64_t stride, int32_t k,
                              float temperature, int32_t type, void *hip_stream)
{
    const char *what = "distill_backward";
    if (const int rc = distill_check(what, logits, idx, val, rows, vocab, stride, k, temperature, type)) return rc;
    REQUIRE_ROWS(what, "dlogits", dlogits, rows, vocab, dlogits_stride, type);
    REQUIRE((dloss && lse) || rows == 0, "%s: dloss or lse is NULL", what);
    REQUIRE(aligned(dloss, 4) && aligned(lse, 4), "%s: dloss and lse must be 4-byte aligned", what);
    if (rows == 0) return COMP_AMS_OK;
    DistillArgs a = {rows, vocab, stride, dlogits_stride, k, temperature, 1.f / temperature, streamed_in(rows * vocab, type), streamed_out(rows * vocab, type), 0};
    with_type(type, [&](auto t) {
        using T = decltype(t);
        if (vocab < kVec<T>) {
            in_launches(rows, kVocabThreads, [&](unsigned first, unsigned count) {
                a.first = first;
                distill_any<T, false, true><<<count, kVocabThreads, 0, static_cast<hipStream_t>(hip_stream)>>>(
                    nullptr, nullptr, static_cast<T *>(dlogits), dloss, static_cast<const T *>(logits), lse, idx, val, a);
            });
            return;
        }
        const int64_t chunk = 4 * 256 * kVec<T>;
        const int64_t pieces = std::max<int64_t>(1, std::min(ceil_div(vocab, 4 * chunk), kMaxBlocks / rows));
        const int64_t len = ceil_div(ceil_div(vocab, pieces), chunk) * chunk;
        const int64_t count = ceil_div(vocab, len);
        in_launches(rows * count, 256, [&](unsigned first, unsigned blocks) {
            a.first = first;
            distill_gradient<T, 256><<<blocks, 256, 0, static_cast<hipStream_t>(hip_stream)>>>(
                static_cast<T *>(dlogits), dloss, static_cast<const T *>(logits), lse, idx, val, a, (int)count, len);
        });
    });
    return launched(what);
}

int comp_ams_distill_grad(float *loss, void *dlogits, const float *dloss, const void *logits, const int32_t *idx, const float *val,
                          int64_t rows, int64_t vocab, int64_t dlogits_stride, int64_t stride, int32_t k, float temperature,
                          int32_t type, void *hip_stream)
{
    const char *what = "distill_grad";
    if (const int rc = distill_check(what, logits, idx, val, rows, vocab, stride, k, temperature, type)) return rc;
    REQUIRE_ROWS(what, "dlogits", dlogits, rows, vocab, dlogits_stride, type);
    REQUIRE(dloss || rows == 0, "%s: dloss is NULL", what);
    REQUIRE(aligned(dloss, 4) && aligned(loss, 4), "%s: dloss and loss must be 4-byte aligned", what);
    if (rows == 0) return COMP_AMS_OK;
    DistillArgs a = {rows, vocab, stride, dlogits_stride, k, temperature, 1.f / temperature, streamed_in(rows * vocab, type), streamed_out(rows * vocab, type), 0};
    with_type(type, [&](auto t) {
        using T = decltype(t);
        auto launch = [&](auto shape) {
            using S = decltype(shape);
            in_launches(rows, S::threads, [&](unsigned first, unsigned count) {
                a.first = first;
                distill_both<T, S::threads, S::vecs, S::sure><<<count, S::threads, 0, static_cast<hipStream_t>(hip_stream)>>>(
                    loss, static_cast<T *>(dlogits), dloss, static_cast<const T *>(logits), idx, val, a);
            });
        };
        const int64_t vecs = ceil_div(vocab, kVec<T>);          // vectors of the row
        if (vocab < kVec<T>)
            in_launches(rows, kVocabThreads, [&](unsigned first, unsigned count) {
                a.first = first;
                distill_any<T, true, true><<<count, kVocabThreads, 0, static_cast<hipStream_t>(hip_stream)>>>(
                    loss, nullptr, static_cast<T *>(dlogits), dloss, static_cast<const T *>(logits), nullptr, idx, val, a);
            });
        else if (vecs <= 256) launch(Shape<256, 1>{});
        else if (vecs <= 512 * 8) with_vecs<512, 1, 8>((int)ceil_div(vecs, 512), launch);
        else if (vecs <= 1024 * 8) with_vecs<1024, 5, 8>((int)ceil_div(vecs, 1024), launch);
        else if (vecs <= 1024 * 12) launch(Shape<1024, 12, 8>{});
        else if (vecs <= 1024 * 16) launch(Shape<1024, 16, 12>{});
        else launch(Shape<1024, 0>{});
    });
    return launched(what);
}

}  // extern "C"
