// The clipped policy loss and the preference loss over rows of logits, with the gradient of the logits.
//
// With x a row, m its maximum, s = sum exp(x - m) and y its token:  l = (x_y - m) - log s;  p = exp(x - m) / s;
// d l / d x = onehot(y) - p.  Either loss is a function of the l alone, so that a row's gradient is slope * (onehot(y) - p)
// with one number, the slope, per row.
//
//   row_stats_kernel     (m, s) of a row, or of a part of one
//   seq_count_kernel, policy_rows_kernel    slope of every row from its sequence's advantage and weight, and its terms of the loss
//   policy_sum_kernel    the terms added up
//   pair_kernel          log ratios of a pair's sequences, the margin, the slopes of the pair's rows
//   pair_sum_kernel      the pairs added up
//   logit_grad_kernel    the gradient, from the row, (m, s) and the slope
//
// Differences x - m are taken before the multiplication by log2(e): rows whose entries all are the type's lowest
// value, or that hold -infinity, come out as their definition has it, and the largest entry's exponential is exactly 1.
#include <cmath>

#include "row_vectors.h"

namespace sr {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr int kRowThreads = 256;
constexpr int kTermThreads = 256;

// exp(x) for x <= 0 by the exponential instruction (results below 2^-126 are 0)
__device__ __forceinline__ float exp_neg(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// running maximum and sum of exponentials relative to it; nothing seen: (-FLT_MAX, 0)
struct RowSum {
    float m, s;
};
__device__ __forceinline__ void merge(RowSum &a, float m2, float s2) {
    const float mn = fmaxf(a.m, m2);
    a.s = a.s * exp_neg(a.m - mn) + s2 * exp_neg(m2 - mn);
    a.m = mn;
}

struct RowArgs {
    const void *logits;
    void *grad;
    int64_t ld_logits, ld_grad;
    const int32_t *targets;
    const uint8_t *mask;
    const int32_t *seq_start;
    float *token_logprob;
    int n_rows, vocab, n_seq, splits, split_elems;
    float grad_scale;
    // workspace
    float2 *part;        // [n_rows][splits] (m, s)
    float *slope;        // [n_rows], grad_scale included
    float4 *terms;       // [n_rows] policy: surrogate, kl, clipped, weight; pairs ([n_seq / 2]): loss, m > 0, rewards
    int32_t *count;      // [n_seq] counting rows
};

// s of a row that does not count
constexpr float kNoRow = -1.f;

// the sequence of a row, or -1: the last one that begins at or before it
__device__ __forceinline__ int sequence_of(const RowArgs &a, int row) {
    int lo = -1, hi = a.n_seq;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.seq_start[mid] <= row) lo = mid;
        else hi = mid;
    }
    return lo >= 0 && row < a.seq_start[lo + 1] ? lo : -1;
}
__device__ __forceinline__ bool row_counts(const RowArgs &a, int row) {
    return (!a.mask || a.mask[row]) && row >= a.seq_start[0] && row < a.seq_start[a.n_seq];
}

template <typename T>
__device__ __forceinline__ float logit_of(const RowArgs &a, int row, int v) {
    return v >= 0 && v < a.vocab ? (float)((const T *)a.logits)[row * a.ld_logits + v] : NAN;
}

// One workgroup per (row, part)
template <typename T>
__global__ __launch_bounds__(kRowThreads) void row_stats_kernel(RowArgs a) {
    constexpr int N = Elem<T>::kPerVec;
    __shared__ RowSum s_part[kRowThreads / 64];
    const int row = blockIdx.x / a.splits, part = blockIdx.x % a.splits;
    float2 *out = a.part + blockIdx.x;
    if (!row_counts(a, row)) {
        if (threadIdx.x == 0) *out = make_float2(0.f, kNoRow);
        return;
    }
    const T *x = (const T *)a.logits + row * a.ld_logits;
    const int from = part * a.split_elems, to = min(from + a.split_elems, a.vocab);
    RowSum r = {-FLT_MAX, 0.f};
    for (int e = from + (int)threadIdx.x * N; e < to; e += kRowThreads * N) {
        float v[N];
        load_widened(x, e, to, -INFINITY, v);
        float mn = r.m;
#pragma unroll
        for (int i = 0; i < N; ++i) mn = fmaxf(mn, v[i]);
        r.s *= exp_neg(r.m - mn);
#pragma unroll
        for (int i = 0; i < N; ++i) r.s += exp_neg(v[i] - mn);
        r.m = mn;
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) merge(r, __shfl_xor(r.m, off, 64), __shfl_xor(r.s, off, 64));
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = r;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kRowThreads / 64; ++w) merge(r, s_part[w].m, s_part[w].s);
        *out = make_float2(r.m, r.s);
    }
}

// (m, s) of a row from its parts, in their order
__device__ __forceinline__ RowSum whole_row(const RowArgs &a, int row) {
    const float2 *p = a.part + (size_t)row * a.splits;
    RowSum r = {p[0].x, p[0].y};
    for (int k = 1; k < a.splits; ++k) merge(r, p[k].x, p[k].y);
    return r;
}

// One workgroup per (row, part), the parts of row_stats_kernel.  In place: a thread reads what it then writes.
template <typename T>
__global__ __launch_bounds__(kRowThreads) void logit_grad_kernel(RowArgs a) {
    constexpr int N = Elem<T>::kPerVec;
    const int row = blockIdx.x / a.splits, part = blockIdx.x % a.splits;
    const T *x = (const T *)a.logits + row * a.ld_logits;
    T *g = (T *)a.grad + row * a.ld_grad;
    const int from = part * a.split_elems, to = min(from + a.split_elems, a.vocab);
    const bool counts = a.part[(size_t)row * a.splits].y != kNoRow;
    if (!counts) {
        const float zero[N] = {};
        for (int e = from + (int)threadIdx.x * N; e < to; e += kRowThreads * N) store_narrowed(g, e, to, zero);
        return;
    }
    const RowSum r = whole_row(a, row);
    const float slope = a.slope[row], f = -slope / r.s;
    const int target = a.targets[row];
    for (int e = from + (int)threadIdx.x * N; e < to; e += kRowThreads * N) {
        float v[N];
        load_widened(x, e, to, -INFINITY, v);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = f * exp_neg(v[i] - r.m);
        if ((unsigned)(target - e) < N)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (target == e + i) v[i] += slope;
        store_narrowed(g, e, to, v);
    }
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

// counting rows of a sequence, a wavefront each
__global__ __launch_bounds__(256) void seq_count_kernel(RowArgs a) {
    const int seq = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (seq >= a.n_seq) return;
    const int from = max(a.seq_start[seq], 0), to = min(a.seq_start[seq + 1], a.n_rows);
    int n = 0;
    if (!a.mask) {
        n = max(to - from, 0);
    } else {
        for (int r = from + lane; r < to; r += 64) n += a.mask[r] != 0;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) n += __shfl_xor(n, off, 64);
    }
    if (lane == 0) a.count[seq] = n;
}

template <typename T>
__global__ __launch_bounds__(kTermThreads) void policy_rows_kernel(RowArgs a, PolicyArgs p) {
    __shared__ int s_rows, s_used;
    if (threadIdx.x == 0) s_rows = s_used = 0;
    __syncthreads();
    int rows = 0, used = 0;
    for (int i = threadIdx.x; i < a.n_seq; i += kTermThreads) {
        rows += a.count[i];
        used += a.count[i] > 0;
    }
    atomicAdd(&s_rows, rows);             // whole numbers: the order does not matter
    atomicAdd(&s_used, used);
    __syncthreads();
    const int row = blockIdx.x * kTermThreads + threadIdx.x;
    if (row >= a.n_rows) return;
    float logprob = 0.f, slope = 0.f;
    float4 term = make_float4(0.f, 0.f, 0.f, 0.f);
    const RowSum r = whole_row(a, row);
    const int seq = r.s == kNoRow ? -1 : sequence_of(a, row);
    if (seq >= 0) {
        logprob = (logit_of<T>(a, row, a.targets[row]) - r.m) - logf(r.s);
        const float w = p.reduce == SR_MEAN_TOKENS      ? 1.f / (float)s_rows
                        : p.reduce == SR_MEAN_SEQUENCES ? 1.f / ((float)s_used * (float)a.count[seq])
                                                        : 1.f / (float)s_used;
        const float A = p.advantages[seq], ratio = expf(logprob - p.old_logprob[row]);
        const float plain = ratio * A, clipped = fminf(fmaxf(ratio, 1.f - p.clip_low), 1.f + p.clip_high) * A;
        const bool out = plain > clipped;
        slope = out ? 0.f : -plain;
        term = make_float4(out ? clipped : plain, 0.f, out ? 1.f : 0.f, w);
        if (p.ref_logprob) {
            const float d = p.ref_logprob[row] - logprob, e = expm1f(d);
            term.y = e - d;
            if (p.kl_coef != 0.f) slope -= p.kl_coef * e;
        }
        slope *= w * a.grad_scale;
    }
    if (a.token_logprob) a.token_logprob[row] = logprob;
    a.slope[row] = slope;
    a.terms[row] = term;
}

constexpr int kSumThreads = 1024;

__global__ __launch_bounds__(kSumThreads) void policy_sum_kernel(RowArgs a, PolicyArgs p) {
    __shared__ double s[kSumThreads / 64];
    double sur = 0.0, kl = 0.0, out = 0.0;
    for (int i = threadIdx.x; i < a.n_rows; i += kSumThreads) {
        const float4 t = a.terms[i];
        if (t.w == 0.f) continue;         // a row that does not count
        sur += (double)t.w * (double)t.x;
        kl += (double)t.w * (double)t.y;
        out += (double)t.w * (double)t.z;
    }
    sur = block_sum<kSumThreads / 64>(sur, s);
    kl = block_sum<kSumThreads / 64>(kl, s);
    out = block_sum<kSumThreads / 64>(out, s);
    if (threadIdx.x == 0) {
        p.stats[0] = (float)((p.kl_coef != 0.f ? (double)p.kl_coef * kl : 0.0) - sur);
        p.stats[1] = (float)sur;
        p.stats[2] = (float)kl;
        p.stats[3] = (float)out;
    }
}

// ---------------------------------------------------------------------------------------------
// preference loss
// ---------------------------------------------------------------------------------------------
struct PairArgs {
    const float *ref_logprob;
    float beta, smoothing;
    float *log_ratio, *stats;
};

// One workgroup per pair.  Rows outside every sequence are left to the first and the last one.
template <typename T>
__global__ __launch_bounds__(kTermThreads) void pair_kernel(RowArgs a, PairArgs p) {
    __shared__ double s[kTermThreads / 64];
    __shared__ float s_slope;
    const int pair = blockIdx.x, pairs = a.n_seq / 2;
    double ratio[2];
    for (int k = 0; k < 2; ++k) {
        const int from = max(a.seq_start[2 * pair + k], 0), to = min(a.seq_start[2 * pair + k + 1], a.n_rows);
        double acc = 0.0;
        for (int row = from + threadIdx.x; row < to; row += kTermThreads) {
            const RowSum r = whole_row(a, row);
            float logprob = 0.f;
            if (r.s != kNoRow) {
                logprob = (logit_of<T>(a, row, a.targets[row]) - r.m) - logf(r.s);
                acc += (double)logprob - (p.ref_logprob ? (double)p.ref_logprob[row] : 0.0);
            }
            if (a.token_logprob) a.token_logprob[row] = logprob;
        }
        ratio[k] = block_sum<kTermThreads / 64>(acc, s);
    }
    if (threadIdx.x == 0) {
        const double reward0 = (double)p.beta * ratio[0], reward1 = (double)p.beta * ratio[1], m = reward0 - reward1;
        const double tail = log1p(exp(-fabs(m)));
        const double sm = p.smoothing;                   // a term with weight 0 is left out: it may be infinite
        const double loss = (sm < 1.0 ? (1.0 - sm) * (fmax(-m, 0.0) + tail) : 0.0) + (sm > 0.0 ? sm * (fmax(m, 0.0) + tail) : 0.0);
        s_slope = (float)((double)p.beta / pairs * (sm / (1.0 + exp(-m)) - (1.0 - sm) / (1.0 + exp(m))) * (double)a.grad_scale);
        if (p.log_ratio) {
            p.log_ratio[2 * pair] = (float)ratio[0];
            p.log_ratio[2 * pair + 1] = (float)ratio[1];
        }
        a.terms[pair] = make_float4((float)loss, m > 0.0 ? 1.f : 0.f, (float)reward0, (float)reward1);
    }
    __syncthreads();
    const int start = max(a.seq_start[2 * pair], 0), mid = a.seq_start[2 * pair + 1], end = min(a.seq_start[2 * pair + 2], a.n_rows);
    for (int row = start + threadIdx.x; row < end; row += kTermThreads) a.slope[row] = row < mid ? s_slope : -s_slope;
    if (a.token_logprob) {
        if (pair == 0)
            for (int row = threadIdx.x; row < min(start, a.n_rows); row += kTermThreads) a.token_logprob[row] = 0.f;
        if (pair == pairs - 1)
            for (int row = max(a.seq_start[a.n_seq], 0) + threadIdx.x; row < a.n_rows; row += kTermThreads) a.token_logprob[row] = 0.f;
    }
}

__global__ __launch_bounds__(kSumThreads) void pair_sum_kernel(RowArgs a, PairArgs p) {
    __shared__ double s[kSumThreads / 64];
    const int pairs = a.n_seq / 2;
    double x[4] = {};
    for (int i = threadIdx.x; i < pairs; i += kSumThreads) {
        const float4 t = a.terms[i];
        x[0] += t.x;
        x[1] += t.y;
        x[2] += t.z;
        x[3] += t.w;
    }
    for (int k = 0; k < 4; ++k) {
        const double sum = block_sum<kSumThreads / 64>(x[k], s);
        if (threadIdx.x == 0) p.stats[k] = (float)(sum / pairs);
    }
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
int check_rows(const sr_token_rows *x, const void *workspace, size_t bytes) {
    if (!x || !workspace || (uintptr_t)workspace % 16) return SR_E_ARG;
    if (x->dtype < SR_F32 || x->dtype > SR_F16 || x->n_rows < 0 || x->vocab < 1 || x->n_seq < 1) return SR_E_ARG;
    if (x->vocab > 1 << 30 || !x->seq_start || !std::isfinite(x->grad_scale)) return SR_E_ARG;
    if (bytes < SR_TOKEN_LOSS_WORKSPACE(x->n_rows, x->n_seq)) return SR_E_ARG;
    if (x->n_rows == 0) return SR_OK;
    const unsigned elem = x->dtype == SR_F32 ? 4 : 2;
    if (!x->logits || (uintptr_t)x->logits % elem || x->ld_logits < x->vocab || !x->targets) return SR_E_ARG;
    if (x->grad && ((uintptr_t)x->grad % elem || x->ld_grad < x->vocab)) return SR_E_ARG;
    return x->grad == x->logits && x->ld_grad != x->ld_logits ? SR_E_ARG : SR_OK;
}

// SR_TOKEN_LOSS_WORKSPACE: 40 bytes a row and 16 a sequence used here, the constant part for the parts of few rows
RowArgs row_args(const sr_token_rows *x, void *workspace) {
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
    char *w = (char *)workspace;
    a.terms = (float4 *)w;                               // 16 bytes a row, or a pair
    w += 16 * ((size_t)x->n_rows + x->n_seq);
    a.part = (float2 *)w;                                // 8 bytes a row, or 48 KiB
    w += 8 * (size_t)x->n_rows + 49152;
    a.slope = (float *)w;
    w += 4 * (size_t)x->n_rows;
    a.count = (int32_t *)w;
    a.splits = 1;
    a.split_elems = x->vocab;
    return a;
}

template <typename F>
int with_type(int dtype, F &&f) {
    if (dtype == SR_F32) return f((float *)nullptr);
    if (dtype == SR_BF16) return f((__bf16 *)nullptr);
    return f((f16_t *)nullptr);
}

template <typename T>
int launch_row_stats(const RowArgs &a, hipStream_t stream) {
    row_stats_kernel<T><<<dim3((unsigned)(a.n_rows * a.splits)), dim3(kRowThreads), 0, stream>>>(a);
    SR_HIP(hipGetLastError());
    return SR_OK;
}
template <typename T>
int launch_logit_grad(const RowArgs &a, hipStream_t stream) {
    logit_grad_kernel<T><<<dim3((unsigned)(a.n_rows * a.splits)), dim3(kRowThreads), 0, stream>>>(a);
    SR_HIP(hipGetLastError());
    return SR_OK;
}

int policy_loss(const sr_token_rows *x, const PolicyArgs &p, void *workspace, hipStream_t stream) {
    RowArgs a = row_args(x, workspace);
    if (x->n_rows > 0)
        SR_TRY(with_type(x->dtype, [&](auto *t) -> int {
            typedef std::remove_pointer_t<decltype(t)> T;
            SR_TRY(launch_row_stats<T>(a, stream));
            seq_count_kernel<<<dim3((a.n_seq + 3) / 4), dim3(256), 0, stream>>>(a);
            SR_HIP(hipGetLastError());
            policy_rows_kernel<T><<<dim3((a.n_rows + kTermThreads - 1) / kTermThreads), dim3(kTermThreads), 0, stream>>>(a, p);
            SR_HIP(hipGetLastError());
            return a.grad ? launch_logit_grad<T>(a, stream) : SR_OK;
        }));
    policy_sum_kernel<<<dim3(1), dim3(kSumThreads), 0, stream>>>(a, p);
    SR_HIP(hipGetLastError());
    return SR_OK;
}

int preference_loss(const sr_token_rows *x, const PairArgs &p, void *workspace, hipStream_t stream) {
    RowArgs a = row_args(x, workspace);
    return with_type(x->dtype, [&](auto *t) -> int {
        typedef std::remove_pointer_t<decltype(t)> T;
        if (a.n_rows > 0) SR_TRY(launch_row_stats<T>(a, stream));
        pair_kernel<T><<<dim3(a.n_seq / 2), dim3(kTermThreads), 0, stream>>>(a, p);
        SR_HIP(hipGetLastError());
        if (a.n_rows > 0 && a.grad) SR_TRY(launch_logit_grad<T>(a, stream));
        pair_sum_kernel<<<dim3(1), dim3(kSumThreads), 0, stream>>>(a, p);
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
    const sr::PolicyArgs p = {old_logprob, ref_logprob, advantages, opt->clip_low, opt->clip_high, opt->kl_coef, opt->reduce, stats};
    return sr::policy_loss(rows, p, workspace, (hipStream_t)stream);
}

extern "C" int sr_preference_loss(const sr_token_rows *rows, const float *ref_logprob, float beta, float label_smoothing,
                                  float *log_ratio, float *stats, void *workspace, size_t workspace_bytes, void *stream) {
    SR_TRY(sr::check_rows(rows, workspace, workspace_bytes));
    if (!stats || rows->n_seq % 2 || !std::isfinite(beta) || !(label_smoothing >= 0.f && label_smoothing <= 1.f)) return SR_E_ARG;
    const sr::PairArgs p = {ref_logprob, beta, label_smoothing, log_ratio, stats};
    return sr::preference_loss(rows, p, workspace, (hipStream_t)stream);
}
