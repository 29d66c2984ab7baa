// Rows over a vocabulary: log probabilities of tokens with entropy and alternatives, and distillation from top lists.
//
//   lse = log sum exp(z / T);  logp = z_t - lse;  entropy = lse - sum p z
//   q = softmax(val / T) over the list;  loss = T^2 sum q (log q - (z / T - lse));  dz = dloss T (exp(z / T - lse) - q)
//
// HBM-bound, with vector instructions close behind where logits have 16 bits: an element costs 8.5 issue slots (widening, maximum,
// fused multiply-add, exponential (two), sum, moment) where HBM leaves about 13.  So rows are read once and held in registers between
// the passes over them, and exponentials are taken as 2^(z log2(e) / T - c) with one fused multiply-add.
// Measured (us of a pass among others, TB/s of what it cannot do without; a copy reaches 6.1, reading alone 6.2): log probabilities with 32
// alternatives 4096 x 100000 bf16 174 (4.7), of which the alternatives 32, 11 of them the join of four pieces; loss and gradient 4096 x 32768
// bf16 113 (4.8); loss 2048 x 50001 f16 39 (5.3); gradient 1024 x 131072 fp32 188 (5.7).
#pragma once
#include "op_common.h"
#include "../../../include/comp_ams_operators.h"

namespace cams_ops {

constexpr int kVocabThreads = 256;
constexpr int kMaxTop = COMP_AMS_MAX_TOP;

template <typename T> constexpr uint32_t kNegInfBits = sizeof(T) == 4 ? 0xff800000u : __is_same(T, bf16_t) ? 0xff80u : 0xfc00u;

// A logit's place in the order of the top list as one whole number: the larger value first, -0 as +0, every NaN above
// +infinity and equal to the others; among equals the lower token.
__device__ __forceinline__ uint32_t order_of(float z)
{
    if (z != z) return 0xffffffffu;
    const uint32_t b = __float_as_uint(z + 0.f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t rank_key(float z, uint32_t token) { return ((uint64_t)order_of(z) << 32) | (uint32_t)~token; }

// Joins the threads' running maxima and sums; every thread receives the row's.  scratch: 2 * kThreads / 64 floats, not to be used again
// before another barrier.
template <int kThreads>
__device__ __forceinline__ Lse block_lse(const Lse &v, float unit, float *scratch)
{
    const float top = team_reduce<MaxOp, kThreads>(v.top, scratch);
    // equal tops first: -infinity beside -infinity is an empty sum, not a NaN
    const float s = v.top == top ? v.sum : v.sum * __builtin_amdgcn_exp2f((v.top - top) * unit);
    return {top, team_reduce<SumOp, kThreads>(s, scratch + kThreads / kWave)};
}

template <int kThreads>
__device__ __forceinline__ uint64_t block_max(uint64_t v, uint64_t *scratch)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = max(v, (uint64_t)__shfl_xor((unsigned long long)v, off, kWave));
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) scratch[threadIdx.x / kWave] = v;
    __syncthreads();
    v = scratch[0];
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) v = max(v, scratch[w]);
    return v;
}

// Rows of any length: the row is read for maximum and sum, for the entropy, and once more for each alternative.
template <typename T>
__global__ __launch_bounds__(kVocabThreads) void logprobs_any(float *__restrict__ logp, float *__restrict__ entropy,
                                                              int32_t *__restrict__ top_idx, float *__restrict__ top_logp,
                                                              const T *__restrict__ logits, const int64_t *__restrict__ tokens,
                                                              int64_t rows, int64_t vocab, int64_t stride, int k)
{
    __shared__ float lse_scratch[2 * kVocabThreads / kWave], scratch[kVocabThreads / kWave];
    __shared__ uint64_t key_scratch[kVocabThreads / kWave];
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T *z = logits + row * stride;
        Lse v = {-INFINITY, 0.f};
        for (int64_t c = threadIdx.x; c < vocab; c += kVocabThreads) v = lse_join(v, {widen1(z[c]), 1.f}, kLog2e);
        v = block_lse<kVocabThreads>(v, kLog2e, lse_scratch);     // the entropy's barrier lies between two of these
        const float log_of = log_sum(v.top, v.sum);
        float w = 0.f;
        for (int64_t c = threadIdx.x; c < vocab; c += kVocabThreads) {
            const float d = widen1(z[c]) - v.top, e = __builtin_amdgcn_exp2f(d * kLog2e);
            if (e != 0.f) w = fmaf(e, d, w);
        }
        w = team_reduce<SumOp, kVocabThreads>(w, scratch);      // block_lse's barriers lie between two of these
        if (threadIdx.x == 0) {
            if (entropy) entropy[row] = log_of - w / v.sum;
            if (logp) {
                const int64_t t = tokens[row];
                logp[row] = t >= 0 && t < vocab ? (widen1(z[t]) - v.top) - log_of : 0.f;
            }
        }
        uint64_t last = ~0ull;
        for (int q = 0; q < k; ++q) {
            uint64_t best = 0;
            for (int64_t c = threadIdx.x; c < vocab; c += kVocabThreads) {
                const uint64_t key = rank_key(widen1(z[c]), (uint32_t)c);
                if (key < last) best = max(best, key);
            }
            last = block_max<kVocabThreads>(best, key_scratch);
            if (threadIdx.x == 0) {
                const uint32_t t = ~(uint32_t)last;
                top_idx[row * k + q] = (int32_t)t;
                top_logp[row * k + q] = (widen1(z[t]) - v.top) - log_of;
            }
        }
    }
}

// The logit of a rank key (-0 comes back as +0).
__device__ __forceinline__ float logit_of(uint64_t key)
{
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}

// Statistics of a piece of a row, in units of log 2 beside the maximum's own: top = max z, sum = sum 2^d, moment = sum 2^d d with
// d = (z - top) log2 e.  The entropy is log sum - moment / sum: no cancellation against lse.
struct Piece {
    float top, sum, moment;
};
__device__ __forceinline__ Piece piece_join(const Piece &a, const Piece &b)
{
    const float top = MaxOp::apply(a.top, b.top);
    const float da = (a.top - top) * kLog2e, db = (b.top - top) * kLog2e;
    const float fa = a.top == top ? 1.f : __builtin_amdgcn_exp2f(da);
    const float fb = b.top == top ? 1.f : __builtin_amdgcn_exp2f(db);
    // an empty piece (top -infinity, sum 0) adds nothing, though its distance is infinite
    const float ma = a.top == top ? a.moment : fa == 0.f ? 0.f : fa * fmaf(da, a.sum, a.moment);
    const float mb = b.top == top ? b.moment : fb == 0.f ? 0.f : fb * fmaf(db, b.sum, b.moment);
    return {top, a.sum * fa + b.sum * fb, ma + mb};
}
// NaN for a row of nothing but -infinity, or with a +infinity (or a NaN, which the sum shows).
__device__ __forceinline__ float piece_entropy(const Piece &p) { return log_sum(p.top, p.sum) - p.moment / p.sum * kLn2; }

constexpr int kMaxPieces = 32;            // of one row; longer vocabularies go to logprobs_any

// Adds the k tokens of the largest keys of z[lo..hi) to the list by bisection over the order and, among the ties at its end,
// over the token; the piece is read once for each bit.  Every thread of the workgroup calls this; hi - lo >= k >= 1.
template <typename T, int kThreads>
__device__ __attribute__((noinline)) void select_slow(const T *z, int64_t lo, int64_t hi, int k, uint64_t *list, uint32_t *count)
{
    __shared__ uint32_t counts[2];
    uint32_t at = 0;
    int turn = 0;
    auto counted = [&](auto &&test) {
        uint32_t mine = 0;
        for (int64_t c = lo + threadIdx.x; c < hi; c += kThreads) mine += test(order_of(widen1(z[c])), (uint32_t)c) ? 1u : 0u;
        if (threadIdx.x == 0) counts[turn] = 0;
        __syncthreads();
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) mine += __shfl_xor(mine, off, kWave);
        if ((threadIdx.x & (kWave - 1)) == 0) atomicAdd(&counts[turn], mine);       // whole numbers: the order does not matter
        __syncthreads();
        const uint32_t all = counts[turn];
        turn ^= 1;
        return all;
    };
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t more = at | (1u << bit);
        if (counted([&](uint32_t o, uint32_t) { return o >= more; }) >= (uint32_t)k) at = more;
    }
    const uint32_t above = counted([&](uint32_t o, uint32_t) { return o > at; });
    const uint32_t ties = (uint32_t)k - above;             // at least one: `at` is the k-th largest
    uint32_t last = 0;                                       // the largest token of which fewer than `ties` ties come before it
    for (int bit = 30; bit >= 0; --bit) {
        const uint32_t more = last | (1u << bit);
        if (counted([&](uint32_t o, uint32_t c) { return o == at && c < more; }) < ties) last = more;
    }
    if (threadIdx.x == 0) *count = 0;
    __syncthreads();
    for (int64_t c = lo + threadIdx.x; c < hi; c += kThreads) {
        const uint32_t o = order_of(widen1(z[c]));
        if (o > at || (o == at && (uint32_t)c <= last)) list[atomicAdd(count, 1u)] = ((uint64_t)o << 32) | (uint32_t)~(uint32_t)c;
    }
    __syncthreads();
}

// The odd rows of a 16-bit array with an odd stride start between two dwords, where 16-byte loads lose a sixth of their rate (6.2 against
// 5.2 TB/s on 1 GB read).  Such a row is read from the element before it, which belongs to the row before or to the space between, and
// which is then ignored.  Returns how many elements that is; the first row of an array is taken as it stands.
template <typename T>
__device__ __forceinline__ int step_back(const T *z, int64_t row)
{
    return sizeof(T) == 2 && row > 0 && (reinterpret_cast<uintptr_t>(z) & 2) ? 1 : 0;
}

// Calls place(key, rank) for each of n keys in LDS with the number of larger ones, where that is below k.  Several lanes share a key
// while there are lanes enough.
template <int kThreads, typename F>
__device__ __forceinline__ void rank_keys(const uint64_t *list, int n, int k, F &&place)
{
    const int lanes = n <= kThreads / 8 ? 8 : n <= kThreads / 4 ? 4 : n <= kThreads / 2 ? 2 : 1;
    const int sub = threadIdx.x & (lanes - 1);
    for (int t = threadIdx.x / lanes; t < n; t += kThreads / lanes) {
        const uint64_t key = list[t];
        int rank = 0;
#pragma unroll 4
        for (int q = sub; q < n; q += lanes) rank += list[q] > key ? 1 : 0;
        for (int off = 1; off < lanes; off <<= 1) rank += __shfl_xor(rank, off, kWave);
        if (sub == 0 && rank < k) place(key, rank);
    }
}

// The k-th largest of `groups` (64, 128 or 256) values in LDS as its place in the order, by one wavefront: bisection over the bits of the
// order, counting by ballots.  kBits: how many of them, from the top, tell values of the type apart in fp32's form: all; those of bfloat16; sign,
// eight bits of exponent (subnormal numbers are normal ones in fp32) and ten of fraction of half precision.
template <typename T> constexpr int kOrderBits = sizeof(T) == 4 ? 32 : __is_same(T, bf16_t) ? 16 : 19;
template <int kBits>
__device__ __forceinline__ uint32_t kth_largest(const float *values, int groups, int k)
{
    const int lane = threadIdx.x & (kWave - 1);
    uint32_t o[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) o[u] = u * kWave < groups ? order_of(values[u * kWave + lane]) : 0u;
    uint32_t at = 0;
    for (int bit = 31; bit > 31 - kBits; --bit) {
        const uint32_t more = at | (1u << bit);
        int n = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) n += __popcll(__ballot(o[u] >= more));
        if (n >= k) at = more;
        if (n == k) break;                       // exactly k reach it: a bound as good as the k-th value itself
    }
    return at;
}

// One piece of a row per workgroup, held in registers between the two looks at it: maximum, sum and moment, and then the
// elements that can be among the k best.  Those are found by a bound: the k-th largest of the maxima of `groups` groups of lanes is
// reached by k elements at least, and by few more (k = 32 of 64 groups: 44 expected).  Vectors that reach it are queued in LDS, their
// elements that do are listed, and the list is ranked by counting.
// A piece is longer than kVecs - 2 slabs (the shape's rule; the last one is shorter than the others by less than a slab).
// With one piece per row the results are final; with more, statistics and keys go to work and logprobs_join follows.
constexpr int kPieceThreads = 512, kPieceVecs = 8;
constexpr int kMaxQueued = 256;           // vectors that reach the bound; more than that (rows of ties) are told apart by select_slow

template <typename T, int kThreads, int kVecs>
__global__ __launch_bounds__(kThreads, kThreads == kPieceThreads ? 8 : 4) void logprobs_regs(float *__restrict__ logp, float *__restrict__ entropy,
                                                          int32_t *__restrict__ top_idx, float *__restrict__ top_logp,
                                                          const T *__restrict__ logits, const int64_t *__restrict__ tokens,
                                                          int64_t vocab, int64_t stride, int k, int groups, int n_pieces,
                                                          int64_t piece_len, int room, Piece *__restrict__ pieces, uint64_t *__restrict__ keys,
                                                          unsigned first)
{
    constexpr int E = kVec<T>, kWaves = kThreads / kWave;
    __shared__ float scratch[kWaves], sum_of[kWaves], moment_of[kWaves], group_max[256];
    __shared__ uint64_t list[kMaxQueued * E];
    __shared__ v4u queue[kMaxQueued];
    __shared__ int queue_at[kMaxQueued];
    __shared__ uint32_t count, queued, strange, bound_order;
    __shared__ float log_sum_lds;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const unsigned block = first + blockIdx.x;           // first: workgroups that earlier launches of the call have taken
    const int64_t row = block / (unsigned)n_pieces, begin = block % (unsigned)n_pieces * piece_len;
    // `back` elements before the row's first one take part in the loads and in nothing else; room: there is a place for one
    const int back = begin == 0 && room ? step_back(logits + row * stride, row) : 0;
    const int64_t lo = begin - back;
    const int len = (int)(min(begin + piece_len, vocab) - lo);
    const T *z = logits + row * stride + lo;
    auto empty = [&](int v) { return v >= kVecs - 2 && (v * kThreads + wave * kWave) * E >= len; };      // nothing for this wavefront
    v4u raw[kVecs];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) raw[v] = load_slab<T, kThreads>(z, v * kThreads * E, tid, len, len, v < kVecs - 2);
    float vec_max[kVecs], top = -INFINITY;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        vec_max[v] = -INFINITY;
        if (empty(v)) continue;
        float x[E];
        settle_slab<T, kThreads>(raw[v], v * kThreads * E, tid, len, len, kNegInfBits<T>, v < kVecs - 2);
        if (v == 0 && back && tid == 0) raw[v][0] = (raw[v][0] & 0xffff0000u) | kNegInfBits<T>;
        widen<T>(raw[v], x);
#pragma unroll
        for (int q = 0; q < E; ++q) vec_max[v] = MaxOp::apply(vec_max[v], x[q]);
        top = MaxOp::apply(top, vec_max[v]);
    }
    // group maxima on the way to the workgroup's
    if (k > 0) {
        const int per = kThreads / groups;
        float g = top;
        for (int off = 1; off < per; off <<= 1) g = MaxOp::apply(g, __shfl_xor(g, off, kWave));
        if ((tid & (per - 1)) == 0) group_max[tid / per] = g;
    }
    if (tid == 0) count = queued = strange = 0;
    const float m = team_reduce<MaxOp, kThreads>(top, scratch);
    const float c = m * kLog2e;
    const bool plain = plain_product(c);
    float s = 0.f, w = 0.f;
    if (plain) {
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            rewiden(raw[v]);
            if (empty(v)) continue;
            float x[E];
            widen<T>(raw[v], x);
#pragma unroll
            for (int q = 0; q < E; ++q) {
                const float d = fmaf(x[q], kLog2e, -c), e = __builtin_amdgcn_exp2f(d);
                s += e;
                w = fmaf(e, fmaxf(d, -1e30f), w);       // an infinite distance has e = 0
            }
            __builtin_amdgcn_sched_barrier(0);          // one vector after the other: few registers, and four workgroups a compute unit
        }
    } else {
#pragma unroll 1
        for (int q = tid + back; q < len; q += kThreads) {     // infinities, or nothing but -infinity and NaN, or large finite masks
            const float x = widen1(z[q]), d = (x - m) * kLog2e, e = x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(d);
            s += e;
            w = fmaf(e, fmaxf(d, -1e30f), w);
        }
    }
    s = lanes_reduce<SumOp, kWave>(s);
    w = lanes_reduce<SumOp, kWave>(w);
    if ((tid & (kWave - 1)) == 0) {
        sum_of[wave] = s;
        moment_of[wave] = w;
        if (!(fabsf(s) < INFINITY)) strange = 1;        // a NaN or an infinity: the bound says nothing then
    }
    if (k > 0 && wave == kWaves - 1) {
        const uint32_t o = kth_largest<kOrderBits<T>>(group_max, groups, k);
        if ((tid & (kWave - 1)) == 0) bound_order = o;
    }
    __syncthreads();
    const bool whole = n_pieces == 1;
    if (wave == 0) {
        const int q = tid & 15;
        Piece piece = {m, lanes_reduce<SumOp, 16>(q < kWaves ? sum_of[q] : 0.f),
                       lanes_reduce<SumOp, 16>(q < kWaves ? moment_of[q] : 0.f)};
        if (plain) {                                    // the moment's distances are off by the same number
            const float f = kept_back(m, kLog2e, c);
            piece.sum *= f;
            piece.moment = fmaf(fmaf(-m, kLog2e, c), piece.sum, piece.moment * f);
        }
        if (tid == 0 && !whole) pieces[block] = piece;
        if (tid == 0 && whole) {
            const float log_of = log_sum(m, piece.sum);
            log_sum_lds = log_of;
            if (entropy) entropy[row] = piece_entropy(piece);
            if (logp) {
                const int64_t t = tokens[row];
                logp[row] = t >= 0 && t < vocab ? (widen1(logits[row * stride + t]) - m) - log_of : 0.f;
            }
        }
    }
    if (k == 0) return;
    float bound = logit_of((uint64_t)bound_order << 32);
    if (bound != bound) bound = -INFINITY;        // places below -infinity's are no number's
    // one atomic a wavefront for all its vectors
    uint64_t reach[kVecs];
    int total = 0;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        reach[v] = __ballot(vec_max[v] >= bound);
        total += __popcll(reach[v]);
    }
    if (total) {
        uint32_t from = 0;
        if ((tid & (kWave - 1)) == 0) from = atomicAdd(&queued, (uint32_t)total);
        from = __builtin_amdgcn_readfirstlane(from);
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            if (reach[v]) {
                const uint32_t slot = from + __builtin_amdgcn_mbcnt_hi((uint32_t)(reach[v] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)reach[v], 0u));
                if (vec_max[v] >= bound && slot < (uint32_t)kMaxQueued) {
                    queue[slot] = raw[v];
                    queue_at[slot] = (v * kThreads + tid) * E;
                }
                from += __popcll(reach[v]);
            }
        }
    }
    __syncthreads();
    if (strange || queued > (uint32_t)kMaxQueued) {
        if (len - back > k) {
            select_slow<T, kThreads>(logits + row * stride, begin, lo + len, k, list, &count);
        } else {
            if (tid == 0) count = (uint32_t)(len - back);
            for (int q = tid + back; q < len; q += kThreads) list[q - back] = rank_key(widen1(z[q]), (uint32_t)(lo + q));
        }
    } else {
        for (int t = tid; t < (int)queued * E; t += kThreads) {
            const int at = queue_at[t / E] + t % E;
            const uint32_t word = queue[t / E][t % E * (int)sizeof(T) / 4];
            float x;
            if constexpr (sizeof(T) == 4) x = __uint_as_float(word);
            else x = widen1(T{(uint16_t)((t & 1) ? word >> 16 : word)});
            if (x >= bound && at >= back && at < len) list[atomicAdd(&count, 1u)] = rank_key(x, (uint32_t)(lo + at));
        }
    }
    __syncthreads();
    const int n = (int)count;
    rank_keys<kThreads>(list, n, k, [&](uint64_t key, int rank) {
        if (whole) {
            top_idx[row * k + rank] = (int32_t)~(uint32_t)key;
            top_logp[row * k + rank] = (logit_of(key) - m) - log_sum_lds;
        } else {
            keys[(int64_t)block * k + rank] = key;
        }
    });
    if (!whole)
        for (int t = n + tid; t < k; t += kThreads) keys[(int64_t)block * k + t] = 0;   // a short last piece
}

// The pieces of a row: statistics joined in order, their best tokens ranked against each other.
template <typename T>
__global__ __launch_bounds__(kVocabThreads) void logprobs_join(float *__restrict__ logp, float *__restrict__ entropy,
                                                               int32_t *__restrict__ top_idx, float *__restrict__ top_logp,
                                                               const T *__restrict__ logits, const int64_t *__restrict__ tokens,
                                                               int64_t vocab, int64_t stride, int k, int n_pieces,
                                                               const Piece *__restrict__ pieces, const uint64_t *__restrict__ keys,
                                                               unsigned first)
{
    extern __shared__ uint64_t list[];
    const int64_t row = first + blockIdx.x;
    const int n = n_pieces * k;
    for (int t = threadIdx.x; t < n; t += kVocabThreads) list[t] = keys[row * n + t];
    Piece p = pieces[row * n_pieces];
    for (int q = 1; q < n_pieces; ++q) p = piece_join(p, pieces[row * n_pieces + q]);
    const float log_of = log_sum(p.top, p.sum);
    if (threadIdx.x == 0) {
        if (entropy) entropy[row] = piece_entropy(p);
        if (logp) {
            const int64_t t = tokens[row];
            logp[row] = t >= 0 && t < vocab ? (widen1(logits[row * stride + t]) - p.top) - log_of : 0.f;
        }
    }
    __syncthreads();
    // every piece's keys are in descending order: a key's rank is its place among its own plus, by bisection, how many of each other
    // piece's are larger
    for (int t = threadIdx.x; t < n; t += kVocabThreads) {
        const uint64_t key = list[t];
        const int own = t / k;
        int rank = t - own * k;
        if (!key) continue;
        for (int q = 0; q < n_pieces; ++q) {
            if (q == own) continue;
            int lo = 0, hi = k;                  // keys [0, lo) are larger, those from hi on are not
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (list[q * k + mid] > key) lo = mid + 1; else hi = mid;
            }
            rank += lo;
        }
        if (rank < k) {
            top_idx[row * k + rank] = (int32_t)~(uint32_t)key;
            top_logp[row * k + rank] = (logit_of(key) - p.top) - log_of;
        }
    }
}

// --- distillation -------------------------------------------------------------------------------------------------

struct DistillArgs {
    int64_t rows, vocab, in_stride, out_stride;
    int32_t k;
    float t, inv_t;          // the temperature and its reciprocal
    bool stream_in, stream_out;
    unsigned first;          // workgroups that earlier launches of the call have taken
};

// The teacher's list of one row, two entries in each lane of a wavefront: every wavefront that needs the list forms its shares for
// itself, without a barrier.
struct Listed {
    int32_t token[2];    // -1: not there
    float q[2];          // the tokens' shares
    float logq[2];       // their logarithms, 0 where the share is 0
    bool any;            // the row lists something
};
static_assert(kMaxTop <= 2 * kWave, "two entries per lane");

// The entries as they are read: loads that may go out before the row's, to be waited for while the row is on its way.
struct RawList {
    int32_t token[2];
    float val[2];
};
__device__ __forceinline__ RawList load_list(const int32_t *__restrict__ idx, const float *__restrict__ val, int64_t row, int k)
{
    const int lane = threadIdx.x & (kWave - 1);
    RawList r;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int t = lane + u * kWave;
        r.token[u] = -1;
        r.val[u] = 0.f;
        if (t < k) {
            r.token[u] = idx[row * k + t];
            r.val[u] = val[row * k + t];
        }
    }
    return r;
}

__device__ __forceinline__ Listed teacher_list(const RawList &r, const DistillArgs &a)
{
    Listed e;
    float v[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const bool there = r.token[u] >= 0 && r.token[u] < a.vocab;
        e.token[u] = there ? r.token[u] : -1;
        v[u] = there ? r.val[u] : -INFINITY;
    }
    e.any = __ballot(e.token[0] >= 0 || e.token[1] >= 0) != 0;
    const float top = lanes_reduce<MaxOp, kWave>(MaxOp::apply(v[0], v[1]));
    float d[2], x[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        d[u] = (v[u] - top) * a.inv_t;           // the difference first: values of any size keep their distances
        // -infinity is listed with nothing, beside others and beside its like
        x[u] = e.token[u] >= 0 && v[u] != -INFINITY ? __builtin_amdgcn_exp2f(d[u] * kLog2e) : 0.f;
    }
    const float sum = lanes_reduce<SumOp, kWave>(x[0] + x[1]), log_sum = logf(sum);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        e.q[u] = x[u] == 0.f ? 0.f : x[u] / sum;
        e.logq[u] = e.q[u] == 0.f ? 0.f : d[u] - log_sum;
    }
    return e;
}

// T^2 sum q (log q - lp) of the row, by one wavefront.
// z: the logits of the lane's entries; v: the row's maximum and sum.
__device__ __forceinline__ float list_loss(const Listed &e, const float (&z)[2], const Lse &v, const DistillArgs &a)
{
    const float log_of = log_sum(v.top, v.sum);
    float part = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u)
        if (e.q[u] != 0.f) part += e.q[u] * (e.logq[u] - fmaf(z[u] - v.top, a.inv_t, -log_of));
    return a.t * a.t * lanes_reduce<SumOp, kWave>(part);
}

// What stands at the listed tokens, by one wavefront: q[u] becomes the sum over the entries that name the token, and token[u] is -1
// but for the first of them.
__device__ __forceinline__ void merge_list(Listed &e, int k)
{
    const int lane = threadIdx.x & (kWave - 1);
    float share[2] = {0.f, 0.f};
    bool first[2] = {true, true};
    for (int t = 0; t < k; ++t) {
        const int u = t >> 6;
        const int32_t token = __builtin_amdgcn_readlane(u ? e.token[1] : e.token[0], t & (kWave - 1));
        const float q = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(u ? e.q[1] : e.q[0]), t & (kWave - 1)));
#pragma unroll
        for (int w = 0; w < 2; ++w)
            if (token == e.token[w]) {
                share[w] += q;
                first[w] = first[w] && t >= lane + w * kWave;
            }
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        e.q[w] = share[w];
        if (!first[w]) e.token[w] = -1;
    }
}

// kVecs vectors of this thread taken into its running maximum and sum.
template <typename T, int kVecs>
__device__ __forceinline__ void take(Lse &v, v4u (&raw)[kVecs], float unit)
{
    constexpr int E = kVec<T>;
    float top = v.top;
#pragma unroll
    for (int r = 0; r < kVecs; ++r) {
        float x[E];
        widen<T>(raw[r], x);
#pragma unroll
        for (int q = 0; q < E; ++q) top = MaxOp::apply(top, x[q]);
    }
    const float from = top == -INFINITY ? 0.f : top;            // nothing but -infinity so far: exponentials of zero, not of NaN
    const float c = from * unit;
    float s = v.sum * __builtin_amdgcn_exp2f((v.top - from) * unit);
#pragma unroll
    for (int r = 0; r < kVecs; ++r) rewiden(raw[r]);
    if (__all(plain_product(c))) {
        float part = 0.f;
#pragma unroll
        for (int r = 0; r < kVecs; ++r) {
            float x[E];
            widen<T>(raw[r], x);
#pragma unroll
            for (int q = 0; q < E; ++q) part += __builtin_amdgcn_exp2f(fmaf(x[q], unit, -c));
        }
        s = fmaf(part, kept_back(from, unit, c), s);
    } else {
#pragma unroll
        for (int r = 0; r < kVecs; ++r) {
            float x[E];
            widen<T>(raw[r], x);
#pragma unroll
            for (int q = 0; q < E; ++q) s += __builtin_amdgcn_exp2f((x[q] - from) * unit);
        }
    }
    v = {top, s};
}

// A row's elements [lo, hi): many(from) for each whole chunk of kVecs slabs, one(from, len) for each slab of what is left.
template <int kSlab, int kVecs, typename Many, typename One>
__device__ __forceinline__ void over_row(int64_t lo, int64_t hi, Many &&many, One &&one)
{
    int64_t from = lo;
    for (; from + (int64_t)kVecs * kSlab <= hi; from += kVecs * kSlab) many(from);
#pragma unroll 1
    for (; from < hi; from += kSlab) one(from, (int)min(hi - from, (int64_t)kSlab));
}

// kVecs slabs of a row from z on, whole ones.
template <typename T, int kThreads, int kVecs>
__device__ __forceinline__ void load_chunk(v4u (&raw)[kVecs], const T *z, bool stream)
{
#pragma unroll
    for (int r = 0; r < kVecs; ++r) raw[r] = load_slab<T, kThreads>(z, r * kThreads * kVec<T>, (int)threadIdx.x, kVecs * kThreads * kVec<T>,
                                                                          kVecs * kThreads * kVec<T>, true, stream);
}
// The gradient of(logit) of kVecs vectors, in slabs of which `len` elements exist.
// All but the first kSure may end inside or lie past it.
template <typename T, int kThreads, int kVecs, int kSure, typename F>
__device__ __forceinline__ void store_chunk(T *out, const v4u (&raw)[kVecs], int len, bool stream, F &&of)
{
    constexpr int E = kVec<T>;
#pragma unroll
    for (int r = 0; r < kVecs; ++r) {
        float x[E];
        widen<T>(raw[r], x);
#pragma unroll
        for (int q = 0; q < E; ++q) x[q] = of(x[q]);
        store_slab<T, kThreads>(out, r * kThreads * E, (int)threadIdx.x, len, narrow<T>(x), r < kSure, stream);
    }
}

// Maximum and sum of a whole row: two sets of vectors, one of them on its way while the other is taken.
template <typename T, int kThreads>
__device__ __forceinline__ Lse take_row(const T *z, int64_t vocab, float unit, bool stream, int back)
{
    constexpr int kVecs = 4, kSlab = kThreads * kVec<T>, kChunk = kVecs * kSlab;
    z -= back;
    vocab += back;
    auto ignore = [&](v4u &raw) {
        if (back && threadIdx.x == 0) raw[0] = (raw[0] & 0xffff0000u) | kNegInfBits<T>;
    };
    Lse v = {-INFINITY, 0.f};
    int64_t from = 0;
    if (vocab >= kChunk) {
        v4u raw[2][kVecs];
        load_chunk<T, kThreads, kVecs>(raw[0], z, stream);
        ignore(raw[0][0]);
        for (;;) {
            from += kChunk;
            bool more = from + kChunk <= vocab;
            if (more) load_chunk<T, kThreads, kVecs>(raw[1], z + from, stream);
            take<T, kVecs>(v, raw[0], unit);
            if (!more) break;
            from += kChunk;
            more = from + kChunk <= vocab;
            if (more) load_chunk<T, kThreads, kVecs>(raw[0], z + from, stream);
            take<T, kVecs>(v, raw[1], unit);
            if (!more) break;
        }
    }
#pragma unroll 1
    for (; from < vocab; from += kSlab) {
        const int len = (int)min(vocab - from, (int64_t)kSlab);
        v4u raw[1] = {load_slab<T, kThreads>(z + from, 0, (int)threadIdx.x, len, len)};
        settle_slab<T, kThreads>(raw[0], 0, (int)threadIdx.x, len, len, kNegInfBits<T>);
        if (from == 0) ignore(raw[0]);
        take<T, 1>(v, raw, unit);
    }
    return v;
}
template <typename T, int kThreads, typename F>
__device__ __forceinline__ void write_row(T *out, const T *z, int64_t lo, int64_t hi, const DistillArgs &a, F &&of)
{
    constexpr int kSlab = kThreads * kVec<T>;
    over_row<kSlab, 4>(
        lo, hi,
        [&](int64_t from) {
            v4u raw[4];
            load_chunk<T, kThreads, 4>(raw, z + from, a.stream_in);
            store_chunk<T, kThreads, 4, 4>(out + from, raw, 4 * kSlab, a.stream_out, of);
        },
        [&](int64_t from, int len) {
            v4u raw[1] = {load_slab<T, kThreads>(z + from, 0, (int)threadIdx.x, len, len)};
            settle_slab<T, kThreads>(raw[0], 0, (int)threadIdx.x, len, len, 0u);
            store_chunk<T, kThreads, 1, 0>(out + from, raw, len, a.stream_out, of);
        });
}

// The loss: one pass over the row with a running maximum and sum, four vectors a thread in flight.  The first wavefront forms the list's
// shares and fetches its logits before the row, so that nothing but a reduction is left when the row is through.
template <typename T, int kThreads>
__global__ __launch_bounds__(kThreads) void distill_forward(float *__restrict__ loss, float *__restrict__ lse_out,
                                                            const T *__restrict__ logits, const int32_t *__restrict__ idx,
                                                            const float *__restrict__ val, DistillArgs a)
{
    __shared__ float lse_scratch[2 * kThreads / kWave];
    const int64_t row = a.first + blockIdx.x;
    const T *z = logits + row * a.in_stride;
    Listed e = {};
    float at[2] = {0.f, 0.f};
    if (threadIdx.x < kWave) {
        e = teacher_list(load_list(idx, val, row, a.k), a);
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (e.token[u] >= 0) at[u] = widen1(z[e.token[u]]);
    }
    Lse v = take_row<T, kThreads>(z, a.vocab, a.inv_t * kLog2e, a.stream_in, step_back(z, row));
    v = block_lse<kThreads>(v, a.inv_t * kLog2e, lse_scratch);
    if (threadIdx.x < kWave) {
        const float l = list_loss(e, at, v, a);
        if (threadIdx.x == 0) {
            if (loss) loss[row] = e.any ? l : 0.f;
            if (lse_out) lse_out[row] = lse_value(v, a.inv_t);
        }
    }
}

// Rows shorter than a vector: one wavefront does them.  kLoss: maximum and sum are formed (else lse is given); kGrad: the gradient is written.
template <typename T, bool kLoss, bool kGrad>
__global__ __launch_bounds__(kVocabThreads) void distill_any(float *__restrict__ loss, float *__restrict__ lse_out, T *dlogits,
                                                             const float *__restrict__ dloss, const T *logits,
                                                             const float *__restrict__ lse_in, const int32_t *__restrict__ idx,
                                                             const float *__restrict__ val, DistillArgs a)
{
    const int64_t row = a.first + blockIdx.x;
    const T *z = logits + row * a.in_stride;
    if (threadIdx.x >= kWave) return;
    Listed e = teacher_list(load_list(idx, val, row, a.k), a);
    float listed[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) listed[u] = e.token[u] >= 0 ? widen1(z[e.token[u]]) : 0.f;
    Lse v = {-INFINITY, 0.f};
    if constexpr (kLoss) {
        for (int c = 0; c < (int)a.vocab; ++c) v = lse_join(v, {widen1(z[c]), 1.f}, a.inv_t * kLog2e);
        const float l = list_loss(e, listed, v, a);
        if (threadIdx.x == 0) {
            if (loss) loss[row] = e.any ? l : 0.f;
            if (lse_out) lse_out[row] = lse_value(v, a.inv_t);
        }
    }
    if constexpr (kGrad) {
        T *out = dlogits + row * a.out_stride;
        const float w = dloss[row] * a.t;
        float p = 0.f, share = 0.f;
        const int lane = threadIdx.x;
        if (lane < (int)a.vocab) {
            const float x = widen1(z[lane]);
            if constexpr (kLoss) p = __builtin_amdgcn_exp2f(fmaf(x - v.top, a.inv_t, -log_sum(v.top, v.sum)) * kLog2e);
            else p = __builtin_amdgcn_exp2f(fmaf(x, a.inv_t, -lse_in[row]) * kLog2e);
        }
        for (int t = 0; t < a.k; ++t) {
            const int32_t token = __builtin_amdgcn_readlane(t < kWave ? e.token[0] : e.token[1], t & (kWave - 1));
            const float q = lane_value(t < kWave ? e.q[0] : e.q[1], t & (kWave - 1));
            if (token == lane) share += q;
        }
        if (lane < (int)a.vocab) out[lane] = narrow1<T>(e.any ? w * (p - share) : 0.f);
    }
}

// The gradient from a given lse: a piece of a row per workgroup.
template <typename T, int kThreads>
__global__ __launch_bounds__(kThreads) void distill_gradient(T *dlogits, const float *__restrict__ dloss, const T *logits,
                                                             const float *__restrict__ lse_in, const int32_t *__restrict__ idx,
                                                             const float *__restrict__ val, DistillArgs a, int n_pieces, int64_t piece_len)
{
    const unsigned block = a.first + blockIdx.x;
    const int64_t row = block / (unsigned)n_pieces, lo = block % (unsigned)n_pieces * piece_len;
    const int64_t hi = min(lo + piece_len, a.vocab);
    const T *z = logits + row * a.in_stride;
    T *out = dlogits + row * a.out_stride;
    const float lse = lse_in[row];
    Listed e = teacher_list(load_list(idx, val, row, a.k), a);
    const float w = dloss[row] * a.t;
    float listed[2] = {0.f, 0.f};
    if (threadIdx.x < kWave) {
        merge_list(e, a.k);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (e.token[u] < lo || e.token[u] >= hi) e.token[u] = -1;
            if (e.token[u] >= 0) listed[u] = widen1(z[e.token[u]]);        // before an in-place gradient replaces it
        }
    }
    __syncthreads();
    if (e.any) write_row<T, kThreads>(out, z, lo, hi, a, [&](float x) { return w * __builtin_amdgcn_exp2f(fmaf(x, a.inv_t, -lse) * kLog2e); });
    else write_row<T, kThreads>(out, z, lo, hi, a, [](float) { return 0.f; });
    __syncthreads();
    if (threadIdx.x < kWave) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (e.token[u] >= 0) {
                const float p = __builtin_amdgcn_exp2f(fmaf(listed[u], a.inv_t, -lse) * kLog2e);
                out[e.token[u]] = narrow1<T>(w * (p - e.q[u]));
            }
    }
}

// Loss and gradient at once.  kVecs > 0: the row stays in registers, kVecs vectors a thread, and is read once.  kVecs = 0: rows of
// any length, read a second time for the gradient.
// The first kSure slabs are known to lie inside the row.
template <typename T, int kThreads, int kVecs, int kSure>
__global__ __launch_bounds__(kThreads, (kThreads <= 512 ? 6 : 4)) void distill_both(float *__restrict__ loss, T *dlogits, const float *__restrict__ dloss,
                                                         const T *logits, const int32_t *__restrict__ idx, const float *__restrict__ val,
                                                         DistillArgs a)
{
    constexpr int E = kVec<T>, kHeld = kVecs ? kVecs : 1;
    __shared__ float lse_scratch[2 * kThreads / kWave];
    const int64_t row = a.first + blockIdx.x;
    const int tid = threadIdx.x;
    const T *z = logits + row * a.in_stride;
    T *out = dlogits + row * a.out_stride;
    const float unit = a.inv_t * kLog2e;
    __shared__ int any_lds;
    const bool first = tid < kWave;
    const float w = dloss[row] * a.t;
    RawList entries = {};
    if (first) entries = load_list(idx, val, row, a.k);
    Lse v = {-INFINITY, 0.f};
    v4u raw[kHeld];
    if constexpr (kVecs > 0) {
#pragma unroll
        for (int r = 0; r < kHeld; ++r) raw[r] = load_slab<T, kThreads>(z, r * kThreads * E, tid, (int)a.vocab, (int)a.vocab, r < kSure, a.stream_in);
    }
    // The first wavefront sees to the list while the row is on its way, and puts it by: beside a row the registers are taken.
    __shared__ int32_t kept_token[2][kWave];
    __shared__ float kept_q[2][kWave], kept_logit[2][kWave], kept_logq[2][kWave];
    if (first) {
        const Listed e = teacher_list(entries, a);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            kept_token[u][tid] = e.token[u];
            kept_q[u][tid] = e.q[u];
            kept_logq[u][tid] = e.logq[u];
            // before an in-place gradient replaces it
            kept_logit[u][tid] = e.token[u] >= 0 ? widen1(z[e.token[u]]) : 0.f;
        }
        if (tid == 0) any_lds = e.any ? 1 : 0;
    }
    if constexpr (kVecs > 0) {
#pragma unroll
        for (int r = 0; r < kHeld; ++r) settle_slab<T, kThreads>(raw[r], r * kThreads * E, tid, (int)a.vocab, (int)a.vocab, kNegInfBits<T>, r < kSure);
        take<T, kHeld>(v, raw, unit);
    } else {
        v = take_row<T, kThreads>(z, a.vocab, unit, false, 0);
    }
    v = block_lse<kThreads>(v, unit, lse_scratch);                         // (its barriers order the list's reads before the writes below)
    const bool any = any_lds != 0;
    const float scale = w / v.sum;
    const float top = v.top, c = v.top * unit;
    const bool plain = plain_product(c);
    const float kept = scale * kept_back(top, unit, c);
    auto usual = [&](float x) { return kept * __builtin_amdgcn_exp2f(fmaf(x, unit, -c)); };
    auto wide = [&](float x) { return scale * __builtin_amdgcn_exp2f((x - top) * unit); };
    auto none = [](float) { return 0.f; };
    if constexpr (kVecs > 0) {
#pragma unroll
        for (int r = 0; r < kHeld; ++r) rewiden(raw[r]);
        if (any && plain) store_chunk<T, kThreads, kHeld, kSure>(out, raw, (int)a.vocab, a.stream_out, usual);
        else if (any) write_row<T, kThreads>(out, z, 0, a.vocab, a, wide);
        else write_row<T, kThreads>(out, z, 0, a.vocab, a, none);
    } else {
        if (any && plain) write_row<T, kThreads>(out, z, 0, a.vocab, a, usual);
        else if (any) write_row<T, kThreads>(out, z, 0, a.vocab, a, wide);
        else write_row<T, kThreads>(out, z, 0, a.vocab, a, none);
    }
    __syncthreads();                                                       // the row is written before its listed tokens are
    if (first) {
        Listed e;
        float listed[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            e.token[u] = kept_token[u][tid];
            e.q[u] = kept_q[u][tid];
            e.logq[u] = kept_logq[u][tid];
            listed[u] = kept_logit[u][tid];
        }
        const float l = list_loss(e, listed, v, a);
        if (tid == 0 && loss) loss[row] = any ? l : 0.f;
        merge_list(e, a.k);
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (e.token[u] >= 0) out[e.token[u]] = narrow1<T>((plain ? usual(listed[u]) : wide(listed[u])) - w * e.q[u]);
    }
}

}  // namespace cams_ops
