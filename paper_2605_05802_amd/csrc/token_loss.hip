// The clipped policy loss and the preference loss over rows of logits, with the gradient of the logits.
//
// With x a row, m its maximum, s = sum exp(x - m) and y its token:  l = (x_y - m) - log s;  p = exp(x - m) / s;
// d l / d x = onehot(y) - p.  Either loss is a function of the l alone, so that a row's gradient is slope * (onehot(y) - p)
// with one number, the slope, per row.
//
// Policy loss with its gradient, rows that fit the registers of a compute unit (token_plan.h):
//   row_info_*           weight and advantage of every row; calls of up to 4096 rows of at most four wavefronts look them up themselves
//   policy_resident_kernel    a row read once, written once
//   policy_sum_kernel    the rows' terms of the loss added up
// Everything else goes through the logits twice:
//   row_stats_kernel     (m, s) of a row, or of a part of one
//   policy_grad_kernel   few rows: the gradient and the loss; without a gradient policy_small_kernel
//   row_info_*, policy_rows_kernel and policy_sum_kernel    the slopes of the rows and the loss
//   pair_grad_kernel     few rows: the gradient and the loss
//   pair_kernel          log ratios of a pair's sequences, the margin, the slopes of the pair's rows
//   logit_grad_kernel    the gradient, from the row, (m, s) and the slope; in passing the pairs added up (pair_sum_kernel without one)
//
// Memory bounds all of them but the smallest calls, which are bound by their two or three launches.  4096 rows of 152064 bf16 (2.49 GB
// read and written): 484 us in policy_resident_kernel, 5.1 TB/s, a large copy's rate; counted reads and writes are those of the
// data.  2048 such rows without a gradient: 95 us in row_stats_kernel, 6.5 TB/s.  16 pairs of 2400 such rows: 126 us in row_stats_kernel and
// 216 in logit_grad_kernel (6.8 TB/s with the memory-side cache's share).
//
// Differences x - m are taken before the multiplication by log2(e): rows whose entries all are the type's lowest
// value, or that hold -infinity, come out as their definition has it, and the largest entry's exponential is exactly 1.
#include <cmath>

#include "row_vectors.h"
#include "token_plan.h"

namespace sr {
namespace {

constexpr int kTermThreads = 256;
constexpr int kSumThreads = 1024;
constexpr int kMostSummedRows = 16384, kShares = 256;      // rows whose terms one workgroup adds; else the workgroups that add them
constexpr int kMostInline = 1024;      // sequences of a small call
constexpr int kMostTableRows = 4096;   // its rows
constexpr int kMostSmallRows = 2048;   // rows whose slopes and terms one workgroup computes
// Pairs, and workgroups, of a call for pair_grad_kernel.  Its wavefronts each go through a pair's rows: 256 rows of 4000 fp32 in 8 pairs
// 10.7 us instead of 12.4, but 64 of 50021 f16, in 12 parts, 16.4 instead of 14.7, and 400 of 1024 fp32 in 16 pairs 13.7 instead of 13.
constexpr int kMostSmallPairs = 8, kMostPairUnits = 256;
static_assert(kMostPairUnits <= kTermThreads, "rows of a pair");
constexpr int kMostAtOnce = 1024;      // workgroups of policy_grad_kernel, all of which run at once (2048 rows of 100000 fp32 in parts of 16 KB: 423 us, with a
                                       // kernel in between 395)
constexpr int kParts = 8192;           // parts of rows that the workspace holds

// exp(x) for x <= 0 by the exponential instruction; results below 2^-126 are 0.
// log2(e) in single precision is 1.33e-8 too small, relative: nothing in a probability, but in a sum of exponentials an error of
// one sign, the same for every row, and a log ratio adds hundreds of rows (150 of them: 2e-5).  The next number up is 6.93e-8 too
// large; thirteen elements of sixteen taken with the one and three with the other are right to 2e-9 on average.
constexpr float kLog2e = 0x1.715476p+0f, kLog2eUp = 0x1.715478p+0f;
static_assert((float)1.44269504088896341 == kLog2e, "the nearest one is the lower one");
__device__ __forceinline__ float exp_neg(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
__device__ __forceinline__ float exp_neg_of_16(float x, int i) { return __builtin_amdgcn_exp2f(x * (i % 5 == 2 ? kLog2eUp : kLog2e)); }

// Running maximum and sum of exponentials relative to it; nothing seen: (-FLT_MAX, 0).  Products and sums that the compiler might
// fuse in one kernel and not in another are written as they are meant: a row comes out the same whichever kernel takes it.
struct RowSum {
    float m, s;
};
__device__ __forceinline__ RowSum one_element(float x) {
    const float m = fmaxf(x, -FLT_MAX);
    return RowSum{m, exp_neg(x - m)};
}
// over a wavefront, or over each 16 lanes of it, in every lane
template <int LANES>
__device__ __forceinline__ RowSum merge_lanes(RowSum r) {
    auto larger = [](float x, float y) { return fmaxf(x, y); };
    auto add = [](float x, float y) { return x + y; };
    const float m = LANES == 16 ? reduce_16(r.m, larger) : reduce_64(r.m, larger), s = r.s * expf(r.m - m);
    return RowSum{m, LANES == 16 ? reduce_16(s, add) : reduce_64(s, add)};
}
// over the wavefronts of a workgroup, in every lane; s: 16 entries of LDS that nobody reads any more
template <int WAVES>
__device__ __forceinline__ RowSum merge_waves(RowSum r, RowSum *s) {
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = r;
    __syncthreads();
    const int w = threadIdx.x & 15;
    return merge_lanes<16>(w < WAVES ? s[w] : RowSum{-FLT_MAX, 0.f});
}
// The elements of COUNT vectors, sixteen at a time
template <typename T, int COUNT>
__device__ __forceinline__ void add_vectors(RowSum &r, const raw16 *raw) {
    constexpr int N = Elem<T>::kPerVec, GROUP = 16 / N;
    static_assert(COUNT % GROUP == 0, "whole groups");
#pragma unroll
    for (int k = 0; k < COUNT; k += GROUP) {
        float v[16], mn = r.m, sum = 0.f;
#pragma unroll
        for (int j = 0; j < GROUP; ++j) Elem<T>::widen(raw[k + j], v + j * N);
#pragma unroll
        for (int i = 0; i < 16; ++i) mn = fmaxf(mn, v[i]);
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += exp_neg_of_16(v[i] - mn, i);
        r.s = fmaf(r.s, exp_neg(r.m - mn), sum);
        r.m = mn;
        __builtin_amdgcn_sched_barrier(0);                   // one group's widened values at a time
    }
}

struct RowArgs {
    const void *logits;
    void *grad;
    int64_t ld_logits, ld_grad;
    const int32_t *targets;
    const uint8_t *mask;
    const int32_t *seq_start;
    float *token_logprob;
    int n_rows, vocab, n_seq;
    int splits, split_elems;           // parts of a row, whole vectors each
    int grad_splits, grad_elems;       // of the gradient's
    int once_units;                    // parts, of the first rows, that are read past the caches (row_stats_kernel)
    float grad_scale;
    // workspace
    float2 *part;        // [n_rows][splits] (m, s)
    float *chosen;       // [n_rows] the logit of the row's token
    float2 *whole;       // [n_rows] (m, s)
    float2 *info;        // [n_rows] policy: weight (0: does not count), advantage
    float *slope;        // [n_rows], grad_scale included
    float4 *terms;       // [n_rows] policy: surrogate, kl, clipped, weight; [n_seq / 2] pairs: loss, m > 0, rewards
    int32_t *count;      // [n_seq + 2] counting rows of the sequences, of all, and the number of sequences that have any
};

// What the gradient reads again stays in the memory-side cache if it was read with default loads, and little else was: the last rows
// of a call are, the others with the non-temporal hint (730 MB of bf16: 118 us, with default loads 130; but the gradient behind
// takes 232 us where all of them were read with the hint, and 215 where none were, or all but the last 384 MB).
constexpr int64_t kKeepBytes = 384 << 20;

// s of a row that does not count
constexpr float kNoRow = -1.f;

__device__ __forceinline__ int row_bound(const RowArgs &a, int row) { return sr::row_bound(row, a.n_rows); }
// A uniform row's mask, by a scalar load of the word that holds it where all of that word is the mask's
__device__ __forceinline__ bool masked_in(const RowArgs &a, int row) {
    if (!a.mask) return true;
    const uintptr_t from = (uintptr_t)a.mask, at = from + row, word = at & ~(uintptr_t)3;
    if (word < from || word + 4 > from + a.n_rows) return a.mask[row] != 0;
    return (read_uniform((const uint32_t *)word) >> (8 * (at & 3)) & 255u) != 0;
}
__device__ __forceinline__ bool row_counts(const RowArgs &a, int row) {
    return row >= read_uniform(a.seq_start) && row < read_uniform(a.seq_start + a.n_seq) && masked_in(a, row);
}

// ---------------------------------------------------------------------------------------------
// streaming: (m, s) in one kernel, the gradient in another
// ---------------------------------------------------------------------------------------------
// The threads and wavefronts of a workgroup for rows of WAVES wavefronts: four rows of one each
constexpr int row_block(int waves) { return waves == 1 ? 256 : 64 * waves; }

// 1 for a row of 16-bit elements that begins inside a word: its vectors begin behind its first element, at a word
template <typename T> __device__ __forceinline__ int inside_word(const T *x) { return sizeof(T) == 2 ? (int)((uintptr_t)x >> 1 & 1) : 0; }
// A part of a row x: whole vectors in [from, full), then single elements to `to`; in front of the first part's one more if the row
// begins inside a word (1701 rows of 50021 bf16 in pairs, a third masked: 77 us, 84 with half of the rows' vectors cutting words).
template <typename T>
struct Part {
    static constexpr int N = Elem<T>::kPerVec;
    int begin, from, full, to;
    __device__ __forceinline__ Part(const T *x, int part, int elems, int vocab) {
        const int first = part * elems, odd = inside_word(x);
        from = first + odd;
        to = min(from + elems, vocab);
        full = from + (to - from) / N * N;
        begin = part ? from : 0;
    }
    // lane t's single element, if that is in front of `to`: those behind the vectors, and one lane more for the first
    __device__ __forceinline__ int single(int t) const { return t == N && begin != from ? begin : full + t; }
};

// The whole vectors of [from, full) of a row, every LANES-th for this thread, four in flight.  ONCE: with the non-temporal hint.
template <typename T, int LANES, bool ONCE>
__device__ __forceinline__ void add_part(RowSum &r, const T *x, int e, int full) {
    constexpr int N = Elem<T>::kPerVec, DEPTH = 4;
    auto load = [&](int j) __attribute__((always_inline)) { return ONCE ? load_vec_once(x + e + j * LANES * N) : load_vec(x + e + j * LANES * N); };
    raw16 raw[DEPTH];
    asm volatile("; once %0" ::"n"((int)ONCE));              // the two forms differ in a hint alone: the compiler would merge them
    for (; e + (DEPTH - 1) * LANES * N < full; e += DEPTH * LANES * N) {
#pragma unroll
        for (int j = 0; j < DEPTH; ++j) raw[j] = load(j);
        add_vectors<T, DEPTH>(r, raw);
    }
    if (e < full) {
#pragma unroll
        for (int j = 0; j < DEPTH; ++j) raw[j] = e + j * LANES * N < full ? load(j) : raw16(Elem<T>::kMinusInf);
        add_vectors<T, DEPTH>(r, raw);
    }
    asm volatile("; once %0" ::"n"((int)ONCE));
}

// WAVES wavefronts per (row, part)
template <typename T, int WAVES>
__global__ __launch_bounds__(row_block(WAVES)) void row_stats_kernel(RowArgs a) {
    constexpr int N = Elem<T>::kPerVec, LANES = 64 * WAVES;
    __shared__ RowSum s_part[16];
    const int unit = WAVES == 1 ? __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)) : blockIdx.x;
    const int t = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    if (unit >= a.n_rows * a.splits) return;                 // wavefronts without a barrier to come, if any
    const int row = unit / a.splits, part = unit - row * a.splits;
    float2 *out = a.part + unit;
    if (!row_counts(a, row)) {
        if (t == 0) *out = make_float2(0.f, kNoRow);
        return;
    }
    const T *x = (const T *)a.logits + row * a.ld_logits;
    const Part<T> q(x, part, a.split_elems, a.vocab);
    const int target = read_uniform(a.targets + row), single = q.single(t);
    RowSum r = {-FLT_MAX, 0.f};
    if (single < q.to) r = one_element((float)x[single]);
    if (unit < a.once_units) add_part<T, LANES, true>(r, x, q.from + t * N, q.full);
    else add_part<T, LANES, false>(r, x, q.from + t * N, q.full);
    // The token's logit for the kernel behind this one: there it would be a cache line and an address translation per row, cold
    const bool holds = target >= q.begin && target < q.to, none = part == 0 && (target < 0 || target >= a.vocab);
    float chosen = NAN;
    if (holds) chosen = (float)x[target];
    r = merge_lanes<64>(r);
    if (WAVES > 1) r = merge_waves<WAVES>(r, s_part);
    if (t == 0) {
        *out = make_float2(r.m, r.s);
        if (holds || none) a.chosen[row] = chosen;
    }
}

// (m, s) of a row from its parts, in their order
__device__ __forceinline__ RowSum whole_row(const RowArgs &a, int row) {
    const float2 *p = a.part + (size_t)row * a.splits;
    if (a.splits == 1 || p[0].y == kNoRow) return RowSum{p[0].x, p[0].y};
    RowSum r = {p[0].x, 0.f};
    for (int k = 1; k < a.splits; ++k) r.m = fmaxf(r.m, p[k].x);
    for (int k = 0; k < a.splits; ++k) r.s = fmaf(p[k].y, expf(p[k].x - r.m), r.s);
    return r;
}
// ... a uniform row's, from at most 64 parts that lie in the lanes, the last one in all lanes behind them
__device__ __forceinline__ RowSum whole_row_of_wave(float2 part, int splits) {
    auto lane = [](float x, int k) __attribute__((always_inline)) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), k)); };
    if (splits == 1 || lane(part.y, 0) == kNoRow) return RowSum{lane(part.x, 0), lane(part.y, 0)};
    RowSum r = {reduce_64(part.x, [](float x, float y) { return fmaxf(x, y); }), 0.f};
    const float e = expf(part.x - r.m);
    for (int k = 0; k < splits; ++k) r.s = fmaf(lane(part.y, k), lane(e, k), r.s);
    return r;
}

// The gradient of the elements of a vector; the row's token is its element number `hot`, if that is one
template <typename T>
__device__ __forceinline__ raw16 gradient(raw16 raw, int hot, float m, float factor, float slope) {
    constexpr int N = Elem<T>::kPerVec;
    float v[N];
    asm volatile("" : "+v"(raw));                            // widened again: what the maximum widened would not fit the registers
    Elem<T>::widen(raw, v);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = factor * exp_neg(v[i] - m);
    if ((unsigned)hot < N)
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (hot == i) v[i] += slope;
    return Elem<T>::narrow(v);
}

// The whole vectors of a part, every LANES-th from e on for this thread
constexpr int kGradDepth = 4;
template <typename T, int LANES>
__device__ __forceinline__ void write_gradient(const T *x, T *g, int e, int full, int target, float m, float factor, float slope) {
    constexpr int N = Elem<T>::kPerVec;
    raw16 raw[kGradDepth];
    for (; e + (kGradDepth - 1) * LANES * N < full; e += kGradDepth * LANES * N) {
#pragma unroll
        for (int j = 0; j < kGradDepth; ++j) raw[j] = load_vec_once(x + e + j * LANES * N);
#pragma unroll
        for (int j = 0; j < kGradDepth; ++j)
            store_vec_once(g + e + j * LANES * N, gradient<T>(raw[j], target - e - j * LANES * N, m, factor, slope));
    }
    for (; e < full; e += LANES * N) store_vec_once(g + e, gradient<T>(load_vec_once(x + e), target - e, m, factor, slope));
}
// ... and its single elements
template <typename T, int LANES>
__device__ __forceinline__ void write_zeros(T *g, const Part<T> &q, int t) {
    for (int e = q.from + t * Elem<T>::kPerVec; e < q.full; e += LANES * Elem<T>::kPerVec) store_vec_once(g + e, raw16(0));
    const int single = q.single(t);
    if (single < q.to) g[single] = (T)0.f;
}
template <typename T>
__device__ __forceinline__ void write_single(const T *x, T *g, const Part<T> &q, int t, int target, float m, float factor, float slope) {
    const int single = q.single(t);
    if (single >= q.to) return;
    const float v = factor * exp_neg((float)x[single] - m);
    g[single] = (T)(target == single ? v + slope : v);
}

// The preference loss
struct PairArgs {
    const float *ref_logprob;
    float beta, smoothing;
    float *log_ratio, *stats;
};

// The mean over pairs of their terms, by a workgroup; s: THREADS / 64 doubles of LDS
template <int THREADS>
__device__ __forceinline__ void sum_pairs(const float4 *terms, int pairs, const PairArgs &p, double *s) {
    double x[4] = {};
    for (int i = threadIdx.x; i < pairs; i += THREADS) {
        const float4 t = terms[i];
        x[0] += t.x;
        x[1] += t.y;
        x[2] += t.z;
        x[3] += t.w;
    }
    for (int k = 0; k < 4; ++k) {
        const double sum = block_sum<THREADS / 64>(x[k], s);
        if (threadIdx.x == 0) p.stats[k] = (float)(sum / pairs);
    }
}

// WAVES wavefronts per (row, part).  In place: a thread reads what it then writes.  p.stats: the first workgroup adds the pairs up.
template <typename T, int WAVES>
__global__ __launch_bounds__(row_block(WAVES)) void logit_grad_kernel(RowArgs a, PairArgs p) {
    constexpr int N = Elem<T>::kPerVec, LANES = 64 * WAVES;
    __shared__ double s[row_block(WAVES) / 64];
    if (p.stats && blockIdx.x == 0) sum_pairs<row_block(WAVES)>(a.terms, a.n_seq / 2, p, s);
    const int unit = WAVES == 1 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    const int t = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    if (unit >= a.n_rows * a.grad_splits) return;
    const int row = unit / a.grad_splits, part = unit - row * a.grad_splits;
    const T *x = (const T *)a.logits + row * a.ld_logits;
    T *g = (T *)a.grad + row * a.ld_grad;
    const Part<T> q(x, part, a.grad_elems, a.vocab);
    const float2 whole = a.whole[row];
    if (whole.y == kNoRow) return write_zeros<T, LANES>(g, q, t);
    const float m = whole.x, slope = a.slope[row], factor = -slope / whole.y;
    const int target = a.targets[row];
    write_single<T>(x, g, q, t, target, m, factor, slope);
    write_gradient<T, LANES>(x, g, q.from + t * N, q.full, target, m, factor, slope);
}

// ---------------------------------------------------------------------------------------------
// policy loss
// ---------------------------------------------------------------------------------------------
struct PolicyArgs {
    const float *old_logprob, *ref_logprob, *advantages;
    float clip_low, clip_high, kl_coef;
    int reduce;
    float *stats;
};

// One bit for every byte of a word that is not zero
__device__ __forceinline__ unsigned set_bytes(unsigned w) {
    const unsigned top = (((w & 0x7f7f7f7fu) + 0x7f7f7f7fu) | w) & 0x80808080u;
    return ((top >> 7) * 0x10204080u) >> 28;                 // bits 0, 8, 16, 24 to 28 .. 31, the other products apart from each other
}
// ... and for sixteen bytes of a mask
__device__ __forceinline__ raw16 load_bytes(const uint8_t *p) {
    typedef uint32_t raw16_bytes __attribute__((ext_vector_type(4), aligned(1)));
    return *(const raw16_bytes *)p;
}
__device__ __forceinline__ unsigned set_bytes_16(raw16 m) {
    return set_bytes(m[0]) | set_bytes(m[1]) << 4 | set_bytes(m[2]) << 8 | set_bytes(m[3]) << 12;
}
// Sums of two whole numbers over the wavefronts of a workgroup, into LDS
__device__ __forceinline__ void add_up(int n, int some, int *rows, int *used) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        n += __shfl_xor(n, off, 64);
        some += __shfl_xor(some, off, 64);
    }
    if ((threadIdx.x & 63) == 0) {
        atomicAdd(rows, n);                                  // whole numbers: the order does not matter
        atomicAdd(used, some);
    }
}

// counting rows of a sequence, a workgroup each
__global__ __launch_bounds__(kTermThreads) void seq_count_kernel(RowArgs a) {
    __shared__ int s_n, s_unused;
    const int seq = blockIdx.x, t = threadIdx.x;
    const int from = row_bound(a, a.seq_start[seq]), to = row_bound(a, a.seq_start[seq + 1]);
    if (!a.mask) {
        if (t == 0) a.count[seq] = max(to - from, 0);
        return;
    }
    if (t == 0) s_n = s_unused = 0;
    __syncthreads();
    int n = 0;
    for (int r = from + 16 * t; r < to; r += 16 * kTermThreads) {
        if (r + 16 <= to) n += __popc(set_bytes_16(load_bytes(a.mask + r)));
        else
            for (int i = r; i < to; ++i) n += a.mask[i] != 0;
    }
    add_up(n, 0, &s_n, &s_unused);
    __syncthreads();
    if (t == 0) a.count[seq] = s_n;
}
// behind the counts of the sequences: their sum, and the number of those that are not 0
__global__ __launch_bounds__(kSumThreads) void seq_total_kernel(RowArgs a) {
    __shared__ int s[2];
    if (threadIdx.x < 2) s[threadIdx.x] = 0;
    __syncthreads();
    int n = 0, some = 0;
    for (int i = threadIdx.x; i < a.n_seq; i += kSumThreads) {
        n += a.count[i];
        some += a.count[i] > 0;
    }
    add_up(n, some, &s[0], &s[1]);
    __syncthreads();
    if (threadIdx.x < 2) a.count[a.n_seq + threadIdx.x] = s[threadIdx.x];
}

// Weight and advantage of a counting row.  count: its sequence's counting rows; rows, used: those of all sequences, and the sequences
// that have any
__device__ __forceinline__ float2 row_info(const PolicyArgs &p, float advantage, int count, int rows, int used) {
    const float w = p.reduce == SR_MEAN_TOKENS      ? 1.f / (float)rows
                    : p.reduce == SR_MEAN_SEQUENCES ? 1.f / ((float)used * (float)count)
                                                    : 1.f / (float)used;
    return make_float2(w, advantage);
}

// The sequences of a small call in LDS.  Counting rows in front of a row: sixteen rows of the mask are a word of bits, with the number
// of set bits before it.
struct SeqTable {
    int start[kMostInline + 1], count[kMostInline], before[kMostTableRows / 16 + 1], rows, used;
    uint16_t bits[kMostTableRows / 16 + 1];
    int wave_total[kMostTableRows / 16 / 64];

    __device__ __forceinline__ int rank(int row) const { return before[row >> 4] + __popc(bits[row >> 4] & ((1u << (row & 15)) - 1u)); }

    // What fill() reads, asked for ahead of it: loads return in order, and those of a row in between would be waited for
    struct Ahead {
        int start;
        raw16 mask;
    };
    static __device__ __forceinline__ Ahead ahead(const RowArgs &a) {
        Ahead x = {};
        const int t = threadIdx.x;
        if (t <= a.n_seq) x.start = a.seq_start[t];
        // the last word's rows are the end of the mask's last sixteen bytes
        if (a.mask && 16 * t < a.n_rows && a.n_rows >= 16) x.mask = load_bytes(a.mask + min(16 * t, a.n_rows - 16));
        return x;
    }

    // by the whole workgroup; barriers inside and behind
    template <int THREADS>
    __device__ __forceinline__ void fill(const RowArgs &a, const Ahead &x) {
        static_assert(kMostTableRows / 16 == 256 && THREADS >= 256, "a word a thread");
        const int t = threadIdx.x;
        if (t <= a.n_seq) start[t] = x.start;
        for (int i = t + THREADS; i <= a.n_seq; i += THREADS) start[i] = a.seq_start[i];
        if (t == 0) rows = used = 0;
        if (a.mask) {
            unsigned mine = 0;
            int ahead = 0;
            if (t < 256) {
                const int n = a.n_rows - 16 * t;
                if (a.n_rows < 16) {
                    for (int i = 0; i < n; ++i) mine |= (unsigned)(a.mask[16 * t + i] != 0) << i;
                } else if (n > 0) {
                    mine = set_bytes_16(x.mask);
                    if (n < 16) mine >>= 16 - n;
                }
                const int own = __popc(mine);
                ahead = own;
#pragma unroll
                for (int off = 1; off < 64; off <<= 1) {
                    const int x = __shfl_up(ahead, off, 64);
                    if ((t & 63) >= off) ahead += x;
                }
                if ((t & 63) == 63) wave_total[t >> 6] = ahead;
                ahead -= own;
            }
            __syncthreads();
            if (t < 256) {
                for (int w = 0; w < t >> 6; ++w) ahead += wave_total[w];
                before[t] = ahead;
                bits[t] = (uint16_t)mine;
                if (t == 255) {
                    before[256] = ahead + __popc(mine);
                    bits[256] = 0;
                }
            }
        }
        __syncthreads();
        int n = 0, some = 0;
        for (int i = t; i < a.n_seq; i += THREADS) {
            const int from = row_bound(a, start[i]), to = row_bound(a, start[i + 1]);
            const int c = from >= to ? 0 : a.mask ? rank(to) - rank(from) : to - from;
            count[i] = c;
            n += c;
            some += c > 0;
        }
        add_up(n, some, &rows, &used);
        __syncthreads();
    }
    __device__ __forceinline__ int sequence(const RowArgs &a, int row) const {
        return !a.mask || bits[row >> 4] >> (row & 15) & 1 ? sequence_of(start, a.n_seq, row) : -1;
    }
    __device__ __forceinline__ float2 info(const RowArgs &a, const PolicyArgs &p, int row) const {
        const int seq = sequence(a, row);
        return seq < 0 ? make_float2(0.f, 0.f) : row_info(p, p.advantages[seq], count[seq], rows, used);
    }
    // of a uniform row
    __device__ __forceinline__ float2 info_of_wave(const RowArgs &a, const PolicyArgs &p, int row) const {
        const int seq = __builtin_amdgcn_readfirstlane(sequence(a, row));
        return seq < 0 ? make_float2(0.f, 0.f) : row_info(p, read_uniform(p.advantages + seq), count[seq], rows, used);
    }
};

__global__ __launch_bounds__(kTermThreads) void row_info_kernel(RowArgs a, PolicyArgs p) {
    const int row = blockIdx.x * kTermThreads + threadIdx.x;
    if (row >= a.n_rows) return;
    const int seq = !a.mask || a.mask[row] ? sequence_of(a.seq_start, a.n_seq, row) : -1;
    a.info[row] = seq < 0 ? make_float2(0.f, 0.f) : row_info(p, p.advantages[seq], a.count[seq], a.count[a.n_seq], a.count[a.n_seq + 1]);
}
// The same three by one workgroup
__global__ __launch_bounds__(kSumThreads) void row_info_small_kernel(RowArgs a, PolicyArgs p) {
    __shared__ SeqTable table;
    table.fill<kSumThreads>(a, SeqTable::ahead(a));
    for (int row = threadIdx.x; row < a.n_rows; row += kSumThreads) a.info[row] = table.info(a, p, row);
}

// A counting row's slope, and its terms of the loss
__device__ __forceinline__ float policy_row(const PolicyArgs &p, float2 info, float logprob, float old_logprob, float ref_logprob,
                                            float4 *term) {
    const float A = info.y, ratio = expf(logprob - old_logprob);
    // an advantage of 0 leaves the row out, also where the ratio is beyond single precision (0 times infinity); NaN stays
    const float plain = A == 0.f && ratio > FLT_MAX ? 0.f : ratio * A;
    const float clipped = fminf(fmaxf(ratio, 1.f - p.clip_low), 1.f + p.clip_high) * A;
    const bool out = plain > clipped;
    float slope = out ? 0.f : -plain;
    *term = make_float4(out ? clipped : plain, 0.f, out ? 1.f : 0.f, info.x);
    if (p.ref_logprob) {
        const float d = ref_logprob - logprob, e = expm1f(d);
        term->y = e <= FLT_MAX ? e - d : e;                  // a token that the policy has given up: infinite, and no difference of infinities
        if (p.kl_coef != 0.f) slope = fmaf(-p.kl_coef, e, slope);
    }
    return slope * info.x;
}

// What a row's slope takes beside its logits
struct RowScalars {
    int target;
    float old_logprob, ref_logprob;
};
__device__ __forceinline__ RowScalars row_scalars(const RowArgs &a, const PolicyArgs &p, int row) {
    return RowScalars{read_uniform(a.targets + row), read_uniform(p.old_logprob + row),
                      p.ref_logprob ? read_uniform(p.ref_logprob + row) : 0.f};
}

struct PolicySums {
    double surrogate = 0.0, kl = 0.0, out = 0.0;
    __device__ __forceinline__ void add(float4 t) {
        if (t.w == 0.f) return;                              // a row that does not count
        surrogate += (double)t.w * (double)t.x;
        kl += (double)t.w * (double)t.y;
        out += (double)t.w * (double)t.z;
    }
    // over a wavefront, into its places in s, 3 * kSumThreads / 64 doubles of LDS
    __device__ __forceinline__ void fold(double *s, int wave) {
        constexpr int WAVES = kSumThreads / 64;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) {
            surrogate += __shfl_xor(surrogate, off, 64);
            kl += __shfl_xor(kl, off, 64);
            out += __shfl_xor(out, off, 64);
        }
        if ((threadIdx.x & 63) == 0) {
            double *mine = s + wave;
            mine[0] = surrogate;
            mine[WAVES] = kl;
            mine[2 * WAVES] = out;
        }
    }
    // over the wavefronts, valid in thread 0
    __device__ __forceinline__ void unfold(const double *s) {
        constexpr int WAVES = kSumThreads / 64;
        __syncthreads();
        if (threadIdx.x >= 64) return;
        const int k = threadIdx.x & (WAVES - 1);             // the first 16 lanes have all they need
        surrogate = s[k];
        kl = s[WAVES + k];
        out = s[2 * WAVES + k];
#pragma unroll
        for (int off = WAVES / 2; off >= 1; off >>= 1) {
            surrogate += __shfl_xor(surrogate, off, 64);
            kl += __shfl_xor(kl, off, 64);
            out += __shfl_xor(out, off, 64);
        }
    }
    __device__ __forceinline__ void gather(double *s) {
        fold(s, threadIdx.x / 64);
        unfold(s);
    }
    __device__ __forceinline__ void finish(const PolicyArgs &p, double *s) {
        gather(s);
        write(p);
    }
    __device__ __forceinline__ void write(const PolicyArgs &p) const {
        if (threadIdx.x != 0) return;
        p.stats[0] = (float)((p.kl_coef != 0.f ? (double)p.kl_coef * kl : 0.0) - surrogate);
        p.stats[1] = (float)surrogate;
        p.stats[2] = (float)kl;
        p.stats[3] = (float)out;
    }
};

// What lies between a row's (m, s) and its gradient: what it reads, and what becomes of that
struct RowInput {
    RowSum r;
    float chosen, old_logprob, ref_logprob;
};
__device__ __forceinline__ RowInput row_input(const RowArgs &a, const PolicyArgs &p, int row) {
    return RowInput{whole_row(a, row), a.chosen[row], p.old_logprob[row], p.ref_logprob ? p.ref_logprob[row] : 0.f};
}
// Its terms of the loss and its log-probability; returns the slope
__device__ __forceinline__ float row_outcome(const RowArgs &a, const PolicyArgs &p, float2 info, const RowInput &in, float4 *term, float *logprob) {
    *logprob = 0.f;
    *term = make_float4(0.f, 0.f, 0.f, 0.f);
    if (info.x == 0.f) return 0.f;
    *logprob = (in.chosen - in.r.m) - logf(in.r.s);
    return policy_row(p, info, *logprob, in.old_logprob, in.ref_logprob, term) * a.grad_scale;
}
__device__ __forceinline__ float4 finish_row(const RowArgs &a, const PolicyArgs &p, int row, float2 info, const RowInput &in) {
    float logprob;
    float4 term;
    const float slope = row_outcome(a, p, info, in, &term, &logprob);
    if (a.token_logprob) a.token_logprob[row] = logprob;
    a.slope[row] = slope;
    a.whole[row] = make_float2(in.r.m, in.r.s);
    return term;
}

__global__ __launch_bounds__(kTermThreads) void policy_rows_kernel(RowArgs a, PolicyArgs p) {
    const int row = blockIdx.x * kTermThreads + threadIdx.x;
    if (row < a.n_rows) a.terms[row] = finish_row(a, p, row, a.info[row], row_input(a, p, row));
}
__global__ __launch_bounds__(kSumThreads) void policy_sum_kernel(RowArgs a, PolicyArgs p) {
    __shared__ double s[3 * kSumThreads / 64];
    PolicySums sums;
    for (int i = threadIdx.x; i < a.n_rows; i += kSumThreads) sums.add(a.terms[i]);
    sums.finish(p, s);
}
// The same in two steps, for more rows than one workgroup adds in the time of a launch: a share of them each, then the shares
__global__ __launch_bounds__(kSumThreads) void policy_share_kernel(RowArgs a, PolicySums *shares) {
    __shared__ double s[3 * kSumThreads / 64];
    PolicySums sums;
    const int each = (a.n_rows + gridDim.x - 1) / gridDim.x, from = blockIdx.x * each, to = min(from + each, a.n_rows);
    for (int i = from + threadIdx.x; i < to; i += kSumThreads) sums.add(a.terms[i]);
    sums.gather(s);
    if (threadIdx.x == 0) shares[blockIdx.x] = sums;
}
__global__ __launch_bounds__(kSumThreads) void policy_shares_kernel(PolicyArgs p, const PolicySums *shares, int n) {
    __shared__ double s[3 * kSumThreads / 64];
    PolicySums sums;
    if ((int)threadIdx.x < n) sums = shares[threadIdx.x];
    sums.finish(p, s);
}

// row_info_*, policy_rows_kernel and policy_sum_kernel by one workgroup: few rows, no gradient
__global__ __launch_bounds__(kSumThreads) void policy_small_kernel(RowArgs a, PolicyArgs p) {
    __shared__ double s[3 * kSumThreads / 64];
    __shared__ SeqTable table;
    constexpr int EACH = kMostSmallRows / kSumThreads;
    const SeqTable::Ahead ahead = SeqTable::ahead(a);
    RowInput in[EACH];                                       // asked for before the table is made
#pragma unroll
    for (int k = 0; k < EACH; ++k)
        if ((int)threadIdx.x + k * kSumThreads < a.n_rows) in[k] = row_input(a, p, threadIdx.x + k * kSumThreads);
    table.fill<kSumThreads>(a, ahead);
    PolicySums sums;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int row = threadIdx.x + k * kSumThreads;
        if (row < a.n_rows) sums.add(finish_row(a, p, row, table.info(a, p, row), in[k]));
    }
    sums.finish(p, s);
}

// The first vectors of a part, asked for while what their gradient takes is worked out
template <typename T, int LANES>
struct EarlyPart {
    static constexpr int N = Elem<T>::kPerVec, COUNT = 12;
    raw16 raw[COUNT];
    __device__ __forceinline__ void load(const T *x, const Part<T> &q, int t) {
#pragma unroll
        for (int j = 0; j < COUNT; ++j)
            if (q.from + j * LANES * N < q.full) raw[j] = load_vec_once(x + min(q.from + (j * LANES + t) * N, q.full - N));    // whole wavefronts
    }
    // the gradient of the whole part
    __device__ __forceinline__ void write(const T *x, T *g, const Part<T> &q, int t, int target, float m, float factor, float slope) {
        int e = q.from + t * N;
        asm volatile("" : "+v"(e));                          // not a path of its own for every number of vectors
        write_single<T>(x, g, q, t, target, m, factor, slope);
#pragma unroll
        for (int j = 0; j < COUNT; ++j) {
            if (e + j * LANES * N < q.full) store_vec_once(g + e + j * LANES * N, gradient<T>(raw[j], target - e - j * LANES * N, m, factor, slope));
            __builtin_amdgcn_sched_barrier(0);               // one vector's widened values at a time
        }
        write_gradient<T, LANES>(x, g, e + COUNT * LANES * N, q.full, target, m, factor, slope);
    }
};

// The gradient of few rows straight from their parts' (m, s): every workgroup works out its row's weight and slope while its first
// vectors are on their way, and one workgroup more, the first, the loss.  Kernels for 128 rows of 152064 fp32: 16 + 24 us, with a
// kernel in between 16 + 6 + 22; 16 rows of 50021 f16 11 us instead of 14 a call.  Four of them a thread instead of twelve: 2 us more, eight: 1.
template <typename T, int WAVES>
__global__ __launch_bounds__(row_block(WAVES)) void policy_grad_kernel(RowArgs a, PolicyArgs p) {
    constexpr int THREADS = row_block(WAVES), N = Elem<T>::kPerVec, LANES = 64 * WAVES;
    __shared__ SeqTable table;
    const SeqTable::Ahead ahead = SeqTable::ahead(a);
    if (blockIdx.x == 0) {
        // as kSumThreads threads would add them up
        __shared__ double s[3 * kSumThreads / 64];
        table.template fill<THREADS>(a, ahead);
        PolicySums sums;
#pragma unroll 1
        for (int k = 0; k < kSumThreads; k += THREADS) {
            sums = PolicySums();
            for (int row = threadIdx.x + k; row < a.n_rows; row += kSumThreads) {
                float logprob;
                float4 term;
                row_outcome(a, p, table.info(a, p, row), row_input(a, p, row), &term, &logprob);
                sums.add(term);
                if (a.token_logprob) a.token_logprob[row] = logprob;
            }
            sums.fold(s, (threadIdx.x + k) / 64);
        }
        sums.unfold(s);
        sums.write(p);
        return;
    }
    const int unit = WAVES == 1 ? __builtin_amdgcn_readfirstlane((blockIdx.x - 1) * 4 + (threadIdx.x >> 6)) : blockIdx.x - 1;
    const int t = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const bool mine = unit < a.n_rows * a.grad_splits;       // false for a wavefront beside others that has nothing left
    const int row = mine ? unit / a.grad_splits : 0, part = mine ? unit - row * a.grad_splits : 0;
    const bool counts = mine && row_counts(a, row);          // a row that does not is not read; asked first: scalar loads are waited for all at once
    __builtin_amdgcn_sched_barrier(0);
    const T *x = (const T *)a.logits + row * a.ld_logits;
    T *g = (T *)a.grad + row * a.ld_grad;
    const Part<T> q(x, part, a.grad_elems, a.vocab);
    const float2 parts = a.part[(size_t)row * a.splits + min((int)threadIdx.x & 63, a.splits - 1)];
    RowInput in = {{}, read_uniform(a.chosen + row), read_uniform(p.old_logprob + row), p.ref_logprob ? read_uniform(p.ref_logprob + row) : 0.f};
    const int target = read_uniform(a.targets + row);
    EarlyPart<T, LANES> early;
    if (counts) early.load(x, q, t);
    table.template fill<THREADS>(a, ahead);
    if (!mine) return;
    const float2 info = table.info_of_wave(a, p, row);
    in.r = whole_row_of_wave(parts, a.splits);
    if (info.x == 0.f || in.r.s == kNoRow) return write_zeros<T, LANES>(g, q, t);
    float logprob;
    float4 term;
    const float slope = row_outcome(a, p, info, in, &term, &logprob);
    early.write(x, g, q, t, target, in.r.m, -slope / in.r.s, slope);
}

// ---------------------------------------------------------------------------------------------
// policy loss with its gradient, a row held in registers between the two
// ---------------------------------------------------------------------------------------------
// WAVES wavefronts take a row, NV vectors a thread: the row is read once and written once.  NV - kGroup vectors of every thread lie
// inside the row, the last kGroup may not.  Rows of one wavefront: four to a workgroup.  LOOP: a workgroup takes every
// gridDim-th row, and asks for the next row's vectors as the gradient's leave the registers.
// TABLE: the workgroups look the weights up for themselves (small calls), else they are in a.info.
template <typename T, int WAVES, int NV, bool LOOP, bool TABLE>
__global__ __launch_bounds__(row_block(WAVES)) void policy_resident_kernel(RowArgs a, PolicyArgs p) {
    static_assert(!(LOOP && TABLE), "a workgroup of many rows reads what row_info_kernel wrote");
    constexpr int N = Elem<T>::kPerVec, LANES = 64 * WAVES, kGroup = 16 / N, SURE = NV - kGroup;
    __shared__ RowSum s_part[2][16];
    const int t = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    int row = WAVES == 1 ? __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)) : blockIdx.x;
    raw16 raw[NV];
    // Loaded unconditionally, from a place in the row, and looked at later: a load under a condition is waited for at its end, and
    // everything before it with it.
    T last, chosen;                                          // a lane's single element, if it has one; the token's
    auto token_at = [&](int target) __attribute__((always_inline)) { return min(max(target, 0), a.vocab - 1); };
    auto part_of = [&](int row) __attribute__((always_inline)) { return Part<T>((const T *)a.logits + row * a.ld_logits, 0, a.vocab, a.vocab); };
    int at = t * N;                                          // the thread's element of the row's first LANES vectors
    auto fetch = [&](int j, const T *x, const Part<T> &q) __attribute__((always_inline)) {
        raw[j] = raw16(Elem<T>::kMinusInf);
        if (j < SURE || at + j * LANES * N < q.full - q.from) raw[j] = load_vec_once(x + q.from + j * LANES * N + (unsigned)at);
    };
    auto put = [&](int j, T *g, const Part<T> &q, raw16 v) __attribute__((always_inline)) {
        if (j < SURE || at + j * LANES * N < q.full - q.from) store_vec_once(g + q.from + j * LANES * N + (unsigned)at, v);
    };
    auto zeros = [&](int row) __attribute__((always_inline)) {
        T *g = (T *)a.grad + row * a.ld_grad;
        const Part<T> q = part_of(row);
        for (int j = 0; j < NV; ++j) put(j, g, q, raw16(0));
        if (q.single(t) < a.vocab) g[q.single(t)] = (T)0.f;
        if (t == 0) {
            if (a.token_logprob) a.token_logprob[row] = 0.f;
            a.terms[row] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
    };
    // the first counting row from `row` on in steps of the grid; those before it get their zeros
    auto counting = [&](int row, float2 *info) __attribute__((always_inline)) {
        for (; row < a.n_rows; row += gridDim.x) {
            *info = read_uniform(a.info + row);
            if (info->x != 0.f) break;
            zeros(row);
        }
        return row;
    };
    float2 info;
    bool mine = row < a.n_rows;                              // false for a wavefront beside others that has no counting row
    SeqTable::Ahead ahead;
    if constexpr (LOOP) {
        row = counting(row, &info);
        if (row >= a.n_rows) return;
    } else if (TABLE) {
        ahead = SeqTable::ahead(a);
        if (mine && !row_counts(a, row)) {
            zeros(row);
            mine = false;
        }
        if (WAVES > 1) {                                     // the workgroup's only row; behind this the number of loads under way is known
            if (!mine) return;
            mine = true;
        }
    } else {
        if (!mine) return;
        info = read_uniform(a.info + row);
        if (info.x == 0.f) return zeros(row);
    }
    const T *x = (const T *)a.logits + row * a.ld_logits;
    Part<T> q = part_of(row);
    if (mine) {
#pragma unroll
        for (int j = 0; j < NV; ++j) fetch(j, x, q);
        last = x[min(q.single(t), a.vocab - 1)];
    }
    RowScalars scalars;
    if (mine) {
        scalars = row_scalars(a, p, row);
        chosen = x[token_at(scalars.target)];
    }
    if constexpr (TABLE) {
        __shared__ SeqTable table;
        table.template fill<row_block(WAVES)>(a, ahead);
        if (!mine) return;
        info = table.info_of_wave(a, p, row);
    }
    RowSum r = {-FLT_MAX, 0.f};
    if (q.single(t) < a.vocab) r = one_element((float)last);
    add_vectors<T, NV>(r, raw);
    if (LOOP) asm volatile("" ::"v"((float)chosen));         // waited for here, so that in the loop nothing but a row's own loads is
    for (int turn = 0;; turn ^= 1) {
        asm volatile("" : "+v"(at));                         // or the loop keeps every vector's address and index in registers
        T *g = (T *)a.grad + row * a.ld_grad;
        float2 next_info;
        const int next = LOOP ? counting(row + gridDim.x, &next_info) : a.n_rows;
        RowScalars next_scalars;
        if (LOOP && next < a.n_rows) next_scalars = row_scalars(a, p, next);
        r = merge_lanes<64>(r);
        // the half of s_part that the row before used may still be read by wavefronts behind this barrier, but not the other
        if (WAVES > 1) r = merge_waves<WAVES>(r, s_part[turn]);
        const float logit = token_at(scalars.target) == scalars.target ? (float)chosen : NAN;
        const float logprob = (logit - r.m) - logf(r.s), m = r.m;
        float4 term;
        const float slope = policy_row(p, info, logprob, scalars.old_logprob, scalars.ref_logprob, &term) * a.grad_scale;
        const float factor = -slope / r.s;
        const int target = scalars.target;
        if (t == 0) {
            if (a.token_logprob) a.token_logprob[row] = logprob;
            a.terms[row] = term;
        }
        const int single = q.single(t);
        if (single < a.vocab) {
            const float v = factor * exp_neg((float)last - m);
            g[single] = (T)(target == single ? v + slope : v);
        }
        const int hot = target - q.from;
        if (next >= a.n_rows) {                              // the same for every wavefront of the row
#pragma unroll
            for (int j = 0; j < NV; ++j) put(j, g, q, gradient<T>(raw[j], hot - at - j * LANES * N, m, factor, slope));
            return;
        }
        // A group of vectors at a time: this row's gradient leaves, the next row's vectors are asked for, and those that were asked
        // for AHEAD vectors earlier are added up, so that neither the memory nor the arithmetic waits for the other.
        constexpr int AHEAD = NV / 2 / kGroup * kGroup;
        x = (const T *)a.logits + next * a.ld_logits;
        const Part<T> next_q = part_of(next);
        last = x[min(next_q.single(t), a.vocab - 1)];
        chosen = x[token_at(next_scalars.target)];
        r = RowSum{-FLT_MAX, 0.f};
#pragma unroll
        for (int k = 0; k < NV; k += kGroup) {
#pragma unroll
            for (int j = k; j < k + kGroup; ++j) {
                put(j, g, q, gradient<T>(raw[j], hot - at - j * LANES * N, m, factor, slope));
                fetch(j, x, next_q);
                __builtin_amdgcn_sched_barrier(0);           // one vector's widened values at a time
            }
            if (k == AHEAD && next_q.single(t) < a.vocab) r = one_element((float)last);
            if (k >= AHEAD) add_vectors<T, kGroup>(r, raw + k - AHEAD);
            __builtin_amdgcn_sched_barrier(0);
        }
        add_vectors<T, AHEAD>(r, raw + NV - AHEAD);
        row = next;
        q = next_q;
        info = next_info;
        scalars = next_scalars;
    }
}

// ---------------------------------------------------------------------------------------------
// preference loss
// ---------------------------------------------------------------------------------------------
// A row's log ratio, and its log-probability; both 0 for one that does not count.  In double: a pair adds hundreds of them, and rounds
// to single precision once.
struct RowRatio {
    double ratio, logprob;
};
__device__ __forceinline__ RowRatio row_ratio(const RowArgs &a, const PairArgs &p, int row, const RowSum &r, float chosen) {
    const double ref = p.ref_logprob ? (double)p.ref_logprob[row] : 0.0;
    if (r.s == kNoRow) return RowRatio{0.0, 0.0};
    const double logprob = (double)(chosen - r.m) - log((double)r.s);
    return RowRatio{logprob - ref, logprob};
}
// A pair's terms of the loss from its sequences' log ratios, and the slope of the preferred one's rows; the other's have its negative
struct PairOutcome {
    float4 term;
    float slope;
};
__device__ __forceinline__ PairOutcome pair_outcome(const RowArgs &a, const PairArgs &p, double ratio0, double ratio1) {
    const double reward0 = (double)p.beta * ratio0, reward1 = (double)p.beta * ratio1;
    // The margin is a difference of sums in double; what becomes of it is good to single precision from there on.
    const float m = (float)(reward0 - reward1), e = expf(-fabsf(m)), tail = log1pf(e), sm = p.smoothing;
    // a term with weight 0 is left out: it may be infinite
    const float loss = (sm < 1.f ? (1.f - sm) * (fmaxf(-m, 0.f) + tail) : 0.f) + (sm > 0.f ? sm * (fmaxf(m, 0.f) + tail) : 0.f);
    const float small = e / (1.f + e), large = 1.f / (1.f + e);      // sigmoid(-|m|), sigmoid(|m|)
    return PairOutcome{make_float4(loss, m > 0.f ? 1.f : 0.f, (float)reward0, (float)reward1),
                       p.beta / (float)(a.n_seq / 2) * (sm * (m >= 0.f ? large : small) - (1.f - sm) * (m >= 0.f ? small : large)) * a.grad_scale};
}

// A workgroup a pair: log ratios, margin, slopes and the pair's terms of the loss.  Rows outside every sequence are left to the first and
// the last pair.
__global__ __launch_bounds__(kTermThreads) void pair_kernel(RowArgs a, PairArgs p) {
    __shared__ double s[kTermThreads / 64], s_ratio[2];
    const int pairs = a.n_seq / 2, pair = blockIdx.x, t = threadIdx.x;
    const int start = row_bound(a, a.seq_start[2 * pair]), end = row_bound(a, a.seq_start[2 * pair + 2]), mid = a.seq_start[2 * pair + 1];
    double ratio[2] = {};
    for (int row = start + t; row < end; row += kTermThreads) {
        const float chosen = a.chosen[row];
        const RowSum r = whole_row(a, row);
        const RowRatio x = row_ratio(a, p, row, r, chosen);
        if (row < mid) ratio[0] += x.ratio;
        else ratio[1] += x.ratio;
        a.whole[row] = make_float2(r.m, r.s);
        if (a.token_logprob) a.token_logprob[row] = (float)x.logprob;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const double sum = block_sum<kTermThreads / 64>(ratio[k], s);
        if (t == 0) s_ratio[k] = sum;
    }
    __syncthreads();
    ratio[0] = s_ratio[0];
    ratio[1] = s_ratio[1];
    const PairOutcome o = pair_outcome(a, p, ratio[0], ratio[1]);
    if (t == 0) {
        a.terms[pair] = o.term;
        if (p.log_ratio) {
            p.log_ratio[2 * pair] = (float)ratio[0];
            p.log_ratio[2 * pair + 1] = (float)ratio[1];
        }
    }
    for (int row = start + t; row < end; row += kTermThreads) a.slope[row] = row < mid ? o.slope : -o.slope;
    auto outside = [&](int row) {
        a.whole[row] = make_float2(0.f, kNoRow);
        if (a.token_logprob) a.token_logprob[row] = 0.f;
    };
    if (pair == 0)
        for (int row = t; row < start; row += kTermThreads) outside(row);
    if (pair == pairs - 1)
        for (int row = end + t; row < a.n_rows; row += kTermThreads) outside(row);
}

// A pair's rows, at most kTermThreads, and their log ratios by one wavefront, added up as pair_kernel's four would.  WRITE: the rows'
// log-probabilities too.
struct PairRows {
    int start, mid, end;
    double ratio[2];
    // starts: seq_start, an entry a lane
    __device__ __forceinline__ PairRows(const RowArgs &a, int starts, int pair)
        : start(row_bound(a, __builtin_amdgcn_readlane(starts, 2 * pair))), mid(__builtin_amdgcn_readlane(starts, 2 * pair + 1)),
          end(row_bound(a, __builtin_amdgcn_readlane(starts, 2 * pair + 2))) {}
    template <bool WRITE>
    __device__ __forceinline__ void add(const RowArgs &a, const PairArgs &p) {
        constexpr int WAVES = kTermThreads / 64;
        double x[WAVES][2] = {};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int row = start + 64 * w + (int)(threadIdx.x & 63);
            if (row >= end) continue;
            const RowRatio one = row_ratio(a, p, row, whole_row(a, row), a.chosen[row]);
            x[w][row < mid ? 0 : 1] = one.ratio;
            if (WRITE && a.token_logprob) a.token_logprob[row] = (float)one.logprob;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            ratio[k] = 0.0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                if (start + 64 * w >= end) continue;         // nothing but zeros
#pragma unroll
                for (int off = 32; off >= 1; off >>= 1) x[w][k] += __shfl_xor(x[w][k], off, 64);
                ratio[k] += x[w][k];
            }
        }
    }
};

// What pair_kernel, logit_grad_kernel and pair_sum_kernel do, for few rows: every wavefront works out the slope of its row's pair while
// the row's first vectors are on their way, and one workgroup more, the first, the loss.  203 rows of 1024 fp32 in 8 pairs: 15 us
// a call with a kernel in between, 12 without; the kernels 3.2 + 6.5 instead of 3.2 + 4.6 + 3.7.
template <typename T, int WAVES>
__global__ __launch_bounds__(row_block(WAVES)) void pair_grad_kernel(RowArgs a, PairArgs p) {
    constexpr int THREADS = row_block(WAVES), LANES = 64 * WAVES;
    const int pairs = a.n_seq / 2, lane = threadIdx.x & 63, starts = a.seq_start[min(lane, a.n_seq)];
    if (blockIdx.x == 0) {
        __shared__ double s[THREADS / 64];
        __shared__ float4 terms[kMostSmallPairs];
        for (int pair = threadIdx.x >> 6; pair < pairs; pair += THREADS / 64) {
            PairRows rows(a, starts, __builtin_amdgcn_readfirstlane(pair));
            rows.template add<true>(a, p);
            if (lane == 0) {
                terms[pair] = pair_outcome(a, p, rows.ratio[0], rows.ratio[1]).term;
                if (p.log_ratio) {
                    p.log_ratio[2 * pair] = (float)rows.ratio[0];
                    p.log_ratio[2 * pair + 1] = (float)rows.ratio[1];
                }
            }
        }
        if (a.token_logprob) {                               // rows outside every sequence
            const int first = row_bound(a, __builtin_amdgcn_readlane(starts, 0)), end = row_bound(a, __builtin_amdgcn_readlane(starts, a.n_seq));
            for (int row = threadIdx.x; row < first; row += THREADS) a.token_logprob[row] = 0.f;
            for (int row = end + threadIdx.x; row < a.n_rows; row += THREADS) a.token_logprob[row] = 0.f;
        }
        __syncthreads();
        sum_pairs<THREADS>(terms, pairs, p, s);
        return;
    }
    const int unit = WAVES == 1 ? __builtin_amdgcn_readfirstlane((blockIdx.x - 1) * 4 + (threadIdx.x >> 6)) : blockIdx.x - 1;
    const int t = WAVES == 1 ? lane : threadIdx.x;
    if (unit >= a.n_rows * a.grad_splits) return;
    const int row = unit / a.grad_splits, part = unit - row * a.grad_splits;
    const bool counts = row_counts(a, row);                  // a row that does not is not read; asked first: scalar loads are waited for all at once
    __builtin_amdgcn_sched_barrier(0);
    const T *x = (const T *)a.logits + row * a.ld_logits;
    T *g = (T *)a.grad + row * a.ld_grad;
    const Part<T> q(x, part, a.grad_elems, a.vocab);
    const float2 parts = a.part[(size_t)row * a.splits + min(lane, a.splits - 1)];
    const int target = read_uniform(a.targets + row);
    EarlyPart<T, LANES> early;
    if (counts) early.load(x, q, t);
    const RowSum r = whole_row_of_wave(parts, a.splits);
    const int seq = __popcll(__ballot(lane < a.n_seq && starts <= row)) - 1;
    if (r.s == kNoRow || seq < 0) return write_zeros<T, LANES>(g, q, t);
    PairRows rows(a, starts, seq >> 1);
    rows.template add<false>(a, p);
    const float of_preferred = pair_outcome(a, p, rows.ratio[0], rows.ratio[1]).slope, slope = row < rows.mid ? of_preferred : -of_preferred;
    early.write(x, g, q, t, target, r.m, -slope / r.s, slope);
}

__global__ __launch_bounds__(kTermThreads) void pair_sum_kernel(RowArgs a, PairArgs p) {
    __shared__ double s[kTermThreads / 64];
    sum_pairs<kTermThreads>(a.terms, a.n_seq / 2, p, s);
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
// Scalar loads drop the low bits of an address
bool whole_words(std::initializer_list<const void *> pointers) {
    for (const void *p : pointers)
        if ((uintptr_t)p % 4) return false;
    return true;
}

// Whether two arrays of n floats share any.  What a row's log-probability is compared with may not be what receives it: in the
// kernels for few rows one workgroup writes while the others still read.
bool overlap(const float *p, const float *q, int n) {
    return p && q && n > 0 && (uintptr_t)p < (uintptr_t)(q + n) && (uintptr_t)q < (uintptr_t)(p + n);
}

int check_rows(const sr_token_rows *x, const void *workspace, size_t bytes) {
    if (!x || !workspace || (uintptr_t)workspace % 16) return SR_E_ARG;
    if (x->dtype < SR_F32 || x->dtype > SR_F16 || x->n_rows < 0 || x->vocab < 1 || x->n_seq < 1) return SR_E_ARG;
    if (x->vocab > 1 << 30 || !x->seq_start || !std::isfinite(x->grad_scale)) return SR_E_ARG;
    if (!whole_words({x->targets, x->seq_start, x->token_logprob})) return SR_E_ARG;
    if (x->n_rows > 1 << 26 || x->n_seq > 1 << 23) return SR_E_LIMIT;     // threads of a launch
    if (bytes < SR_TOKEN_LOSS_WORKSPACE(x->n_rows, x->n_seq)) return SR_E_ARG;
    if (x->n_rows == 0) return SR_OK;
    const unsigned elem = x->dtype == SR_F32 ? 4 : 2;
    if (!x->logits || (uintptr_t)x->logits % elem || x->ld_logits < x->vocab || !x->targets) return SR_E_ARG;
    if (x->grad && ((uintptr_t)x->grad % elem || x->ld_grad < x->vocab)) return SR_E_ARG;
    return x->grad == x->logits && x->ld_grad != x->ld_logits ? SR_E_ARG : SR_OK;
}

// SR_TOKEN_LOSS_WORKSPACE: of every row 16 bytes of terms, 8 each of (m, s) as parts, whole, and of weight and advantage, 4 each of
// slope and the token's logit;
// of every sequence 16 (a pair's terms) and 4; the constant part for more parts than rows
RowArgs row_args(const sr_token_rows *x, const RowPlan &plan, void *workspace) {
    RowArgs a{};
    a.logits = x->logits;
    a.grad = x->grad;
    a.ld_logits = x->ld_logits;
    a.ld_grad = x->ld_grad;
    a.targets = x->targets;
    a.mask = x->mask;
    a.seq_start = x->seq_start;
    a.token_logprob = x->token_logprob;
    a.n_rows = x->n_rows;
    a.vocab = x->vocab;
    a.n_seq = x->n_seq;
    a.grad_scale = x->grad_scale;
    const size_t rows = (size_t)x->n_rows;
    char *w = (char *)workspace;
    auto take = [&](size_t bytes) {
        char *p = w;
        w += bytes;
        return p;
    };
    a.terms = (float4 *)take(16 * (rows + x->n_seq));
    a.part = (float2 *)take(8 * (rows > kParts ? rows : kParts));
    a.whole = (float2 *)take(8 * rows);
    a.info = (float2 *)take(8 * rows);
    a.slope = (float *)take(4 * rows);
    a.chosen = (float *)take(4 * rows);
    a.count = (int32_t *)take(4 * ((size_t)x->n_seq + 2));
    a.splits = plan.parts;
    a.split_elems = plan.elems;
    const int units = a.n_rows * a.splits;
    const int64_t kept = kKeepBytes / ((int64_t)a.split_elems * (x->dtype == SR_F32 ? 4 : 2));
    a.once_units = !a.grad ? units : kept < units ? units - (int)kept : 0;
    a.grad_splits = plan.grad_parts;
    a.grad_elems = plan.grad_elems;
    return a;
}

template <typename F>
int with_type(int dtype, F &&f) {
    if (dtype == SR_F32) return f((float *)nullptr);
    if (dtype == SR_BF16) return f((__bf16 *)nullptr);
    return f((f16_t *)nullptr);
}

template <typename T>
int launch_row_stats(const RowArgs &a, int waves, hipStream_t stream) {
    const int units = a.n_rows * a.splits;
    if (waves == 1) row_stats_kernel<T, 1><<<dim3(ceil_div(units, 4)), dim3(row_block(1)), 0, stream>>>(a);
    else if (waves == 4) row_stats_kernel<T, 4><<<dim3(units), dim3(row_block(4)), 0, stream>>>(a);
    else row_stats_kernel<T, 16><<<dim3(units), dim3(row_block(16)), 0, stream>>>(a);
    SR_HIP(hipGetLastError());
    return SR_OK;
}
template <typename T>
int launch_logit_grad(const RowArgs &a, const PairArgs &p, int waves, hipStream_t stream) {
    const int units = a.n_rows * a.grad_splits;
    if (waves == 1) logit_grad_kernel<T, 1><<<dim3(ceil_div(units, 4)), dim3(row_block(1)), 0, stream>>>(a, p);
    else logit_grad_kernel<T, 4><<<dim3(units), dim3(row_block(4)), 0, stream>>>(a, p);
    SR_HIP(hipGetLastError());
    return SR_OK;
}

template <typename T>
int launch_pair_grad(const RowArgs &a, const PairArgs &p, int waves, hipStream_t stream) {
    const int units = a.n_rows * a.grad_splits;
    if (waves == 1) pair_grad_kernel<T, 1><<<dim3(ceil_div(units, 4) + 1), dim3(row_block(1)), 0, stream>>>(a, p);
    else pair_grad_kernel<T, 4><<<dim3(units + 1), dim3(row_block(4)), 0, stream>>>(a, p);
    SR_HIP(hipGetLastError());
    return SR_OK;
}
template <typename T>
int launch_policy_grad(const RowArgs &a, const PolicyArgs &p, int waves, hipStream_t stream) {
    const int units = a.n_rows * a.grad_splits;
    if (waves == 1) policy_grad_kernel<T, 1><<<dim3(ceil_div(units, 4) + 1), dim3(row_block(1)), 0, stream>>>(a, p);
    else policy_grad_kernel<T, 4><<<dim3(units + 1), dim3(row_block(4)), 0, stream>>>(a, p);
    SR_HIP(hipGetLastError());
    return SR_OK;
}

int launch_row_info(const RowArgs &a, const PolicyArgs &p, hipStream_t stream) {
    if (a.n_seq <= kMostInline && a.n_rows <= kMostTableRows) {
        row_info_small_kernel<<<dim3(1), dim3(kSumThreads), 0, stream>>>(a, p);
        SR_HIP(hipGetLastError());
        return SR_OK;
    }
    seq_count_kernel<<<dim3(a.n_seq), dim3(kTermThreads), 0, stream>>>(a);
    SR_HIP(hipGetLastError());
    seq_total_kernel<<<dim3(1), dim3(kSumThreads), 0, stream>>>(a);
    SR_HIP(hipGetLastError());
    row_info_kernel<<<dim3(ceil_div(a.n_rows, kTermThreads)), dim3(kTermThreads), 0, stream>>>(a, p);
    SR_HIP(hipGetLastError());
    return SR_OK;
}

// vecs: vectors of a thread; the kernels have whole groups of them
template <typename T, int WAVES, int NV>
int launch_resident(const RowArgs &a, const PolicyArgs &p, int vecs, hipStream_t stream) {
    constexpr int kGroup = 16 / Elem<T>::kPerVec;
    if constexpr (NV + kGroup <= (WAVES == 1 ? kMostOneWave : kMostResident))
        if (vecs > NV) return launch_resident<T, WAVES, NV + kGroup>(a, p, vecs, stream);
    if constexpr (WAVES == 16) {
        SR_TRY(launch_row_info(a, p, stream));
        policy_resident_kernel<T, WAVES, NV, true, false><<<dim3(a.n_rows < 256 ? a.n_rows : 256), dim3(row_block(WAVES)), 0, stream>>>(a, p);
    } else {
        const int blocks = WAVES == 1 ? ceil_div(a.n_rows, 4) : a.n_rows;
        if (a.n_seq <= kMostInline && a.n_rows <= kMostTableRows) {
            policy_resident_kernel<T, WAVES, NV, false, true><<<dim3(blocks), dim3(row_block(WAVES)), 0, stream>>>(a, p);
        } else {
            SR_TRY(launch_row_info(a, p, stream));
            policy_resident_kernel<T, WAVES, NV, false, false><<<dim3(blocks), dim3(row_block(WAVES)), 0, stream>>>(a, p);
        }
    }
    SR_HIP(hipGetLastError());
    return SR_OK;
}
template <typename T>
int launch_resident(const RowArgs &a, const PolicyArgs &p, int waves, int vecs, hipStream_t stream) {
    if (waves == 1) return launch_resident<T, 1, 16 / Elem<T>::kPerVec>(a, p, vecs, stream);
    if (waves == 4) return launch_resident<T, 4, 4>(a, p, vecs, stream);
    return launch_resident<T, 16, 4>(a, p, vecs, stream);
}

int policy_loss(const sr_token_rows *x, const PolicyArgs &p, void *workspace, hipStream_t stream) {
    const RowPlan plan = plan_policy_rows(x->n_rows, x->vocab, x->dtype == SR_F32 ? 4 : 2);
    if (!launches_fit(plan, x->n_rows, x->grad != nullptr)) return SR_E_LIMIT;
    const RowArgs a = row_args(x, plan, workspace);
    const bool small = a.n_rows <= kMostSmallRows && a.n_seq <= kMostInline && !(a.grad && plan.resident);
    if (a.n_rows > 0)
        SR_TRY(with_type(x->dtype, [&](auto *t) -> int {
            typedef std::remove_pointer_t<decltype(t)> T;
            if (a.grad && plan.resident) return launch_resident<T>(a, p, plan.waves, plan.resident, stream);
            SR_TRY(launch_row_stats<T>(a, plan.waves, stream));
            if (small && a.grad && a.n_rows * a.grad_splits <= kMostAtOnce) return launch_policy_grad<T>(a, p, plan.grad_waves, stream);
            if (small) {
                policy_small_kernel<<<dim3(1), dim3(kSumThreads), 0, stream>>>(a, p);
                SR_HIP(hipGetLastError());
            } else {
                SR_TRY(launch_row_info(a, p, stream));
                policy_rows_kernel<<<dim3(ceil_div(a.n_rows, kTermThreads)), dim3(kTermThreads), 0, stream>>>(a, p);
                SR_HIP(hipGetLastError());
            }
            return a.grad ? launch_logit_grad<T>(a, PairArgs{}, plan.grad_waves, stream) : SR_OK;
        }));
    if (a.n_rows > 0 && small) return SR_OK;
    if (a.n_rows > kMostSummedRows) {
        PolicySums *shares = (PolicySums *)a.part;           // 64 KiB at least, and no longer read
        policy_share_kernel<<<dim3(kShares), dim3(kSumThreads), 0, stream>>>(a, shares);
        SR_HIP(hipGetLastError());
        policy_shares_kernel<<<dim3(1), dim3(kSumThreads), 0, stream>>>(p, shares, kShares);
    } else {
        policy_sum_kernel<<<dim3(1), dim3(kSumThreads), 0, stream>>>(a, p);
    }
    SR_HIP(hipGetLastError());
    return SR_OK;
}

int preference_loss(const sr_token_rows *x, const PairArgs &p, void *workspace, hipStream_t stream) {
    const RowPlan plan = plan_streamed_rows(x->n_rows, x->vocab, x->dtype == SR_F32 ? 4 : 2);
    if (!launches_fit(plan, x->n_rows, x->grad != nullptr)) return SR_E_LIMIT;
    const RowArgs a = row_args(x, plan, workspace);
    return with_type(x->dtype, [&](auto *t) -> int {
        typedef std::remove_pointer_t<decltype(t)> T;
        if (a.n_rows > 0) SR_TRY(launch_row_stats<T>(a, plan.waves, stream));
        if (a.grad && a.n_rows > 0 && a.n_seq <= 2 * kMostSmallPairs && a.n_rows * a.grad_splits <= kMostPairUnits)
            return launch_pair_grad<T>(a, p, plan.grad_waves, stream);
        pair_kernel<<<dim3(a.n_seq / 2), dim3(kTermThreads), 0, stream>>>(a, p);
        SR_HIP(hipGetLastError());
        if (a.n_rows > 0 && a.grad) return launch_logit_grad<T>(a, p, plan.grad_waves, stream);
        pair_sum_kernel<<<dim3(1), dim3(kTermThreads), 0, stream>>>(a, p);
        SR_HIP(hipGetLastError());
        return SR_OK;
    });
}

}  // namespace
}  // namespace sr

extern "C" int sr_policy_loss(const sr_token_rows *rows, const float *old_logprob, const float *ref_logprob, const float *advantages,
                              const sr_policy_options *opt, float *stats, void *workspace, size_t workspace_bytes, void *stream) {
    SR_TRY(sr::check_rows(rows, workspace, workspace_bytes));
    if (!opt || !stats || !advantages || (rows->n_rows > 0 && !old_logprob)) return SR_E_ARG;
    if (!(opt->clip_low >= 0.f && opt->clip_low <= 1.f) || !(opt->clip_high >= 0.f) || !std::isfinite(opt->clip_high)) return SR_E_ARG;
    if (!std::isfinite(opt->kl_coef) || (opt->kl_coef != 0.f && !ref_logprob && rows->n_rows > 0)) return SR_E_ARG;
    if (opt->reduce < SR_MEAN_TOKENS || opt->reduce > SR_MEAN_SUMS) return SR_E_ARG;
    if (!sr::whole_words({old_logprob, ref_logprob, advantages, stats})) return SR_E_ARG;
    for (const float *in : {old_logprob, ref_logprob})
        if (sr::overlap(rows->token_logprob, in, rows->n_rows)) return SR_E_ARG;
    const sr::PolicyArgs p = {old_logprob, ref_logprob, advantages, opt->clip_low, opt->clip_high, opt->kl_coef, opt->reduce, stats};
    return sr::policy_loss(rows, p, workspace, (hipStream_t)stream);
}

extern "C" int sr_preference_loss(const sr_token_rows *rows, const float *ref_logprob, float beta, float label_smoothing,
                                  float *log_ratio, float *stats, void *workspace, size_t workspace_bytes, void *stream) {
    SR_TRY(sr::check_rows(rows, workspace, workspace_bytes));
    if (!sr::whole_words({ref_logprob, log_ratio, stats}) || sr::overlap(rows->token_logprob, ref_logprob, rows->n_rows)) return SR_E_ARG;
    if (!stats || rows->n_seq % 2 || !std::isfinite(beta) || !(label_smoothing >= 0.f && label_smoothing <= 1.f)) return SR_E_ARG;
    const sr::PairArgs p = {ref_logprob, beta, label_smoothing, log_ratio, stats};
    return sr::preference_loss(rows, p, workspace, (hipStream_t)stream);
}
