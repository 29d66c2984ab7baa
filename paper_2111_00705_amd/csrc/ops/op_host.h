// Host-side helpers of the operators in this folder: errors, checks of arguments, launches, constants chosen from sizes as types.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../../include/comp_ams_operators.h"
#include "op_common.h"
#include "op_sizes.h"

namespace cams_ops {

inline thread_local char g_error[512] = "";      // one message for the calls of all files

inline int fail(int code, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_error, sizeof g_error, fmt, ap);
    va_end(ap);
    return code;
}

// The status of the launches since the runtime's "last error" was clear; it is cleared again, or the caller's next HIP call
// would trip over it.
inline int launched(const char *what)
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

inline bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

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
inline bool streamed_out(int64_t elements, int32_t type) { return elements > ((int64_t)80 << 20) / (int64_t)type_size(type); }
inline bool streamed_in(int64_t elements, int32_t type) { return elements > ((int64_t)256 << 20) / (int64_t)type_size(type); }

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

}  // namespace cams_ops
