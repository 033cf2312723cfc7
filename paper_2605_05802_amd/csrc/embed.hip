// Embedding: rows of a table for a list of tokens, scaled, and the gradient of the table.
//
// out[i] = scale * table[token i]; d_table[v] [+]= scale * sum of d_out[i] over the i whose token is v, in ascending order of i, so that
// the sums are the same bit for bit from call to call.  Tokens outside the vocabulary have a row of zeros and no gradient.
// Memory bounds both; of a whole table's gradient most is zeros to write.
//
// The gradient sorts (token, i) by counting, for every i, how many come before it.  The sorted list is cut into chunks of equal length whatever
// tokens they hold, so that a token of half the batch is as well spread as any: a wavefront adds up a chunk's rows, 64 vectors of columns, and
// writes the sums of the tokens that lie in its chunk alone; sums of tokens that reach over an end go to the workspace, and a second kernel
// adds those up, chunk by chunk.
#include <cmath>

#include "row_ops.h"

namespace sr {
namespace {

// ---------------------------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------------------------
struct EmbedArgs {
    const void *table;
    void *out;
    const int32_t *tokens;
    int64_t ld_table, ld_out;
    int n, vocab, width, parts;      // parts: workgroups of a row, 256 vectors each
    FastDiv by_parts;
    int lanes_shift;                 // log2 of the threads of a row where several rows share a workgroup
    float scale;
};

template <typename T, typename O, int N>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a) {
    int row, v;
    if (a.parts > 1) {
        row = quotient(blockIdx.x, a.by_parts);
        v = (int)(blockIdx.x - (unsigned)row * a.parts) * 256 + threadIdx.x;
    } else {
        row = (int)((blockIdx.x << (8 - a.lanes_shift)) + (threadIdx.x >> a.lanes_shift));
        v = threadIdx.x & ((1 << a.lanes_shift) - 1);
    }
    if (row >= a.n) return;
    const Span s = span_of<N>(v, a.width);
    if (s.skip == N) return;
    const int token = a.tokens[row];
    float x[N];
    if ((unsigned)token < (unsigned)a.vocab) {
        Part<T, N> p;
        p.load((const T *)a.table + token * a.ld_table + s.c);
        p.widen(x);
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] *= a.scale;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = 0.f;
    }
    store_span<N>((O *)a.out + row * a.ld_out, s, x);
}

template <typename T, typename O, int N>
int launch_embed(EmbedArgs a, hipStream_t stream) {
    const int vecs = ceil_div(a.width, N);
    a.parts = ceil_div(vecs, 256);
    a.by_parts = fast_div(a.parts);
    a.lanes_shift = 0;
    while ((1 << a.lanes_shift) < vecs && a.lanes_shift < 8) ++a.lanes_shift;
    const int64_t blocks = a.parts > 1 ? (int64_t)a.n * a.parts : ((int64_t)a.n + (256 >> a.lanes_shift) - 1) >> (8 - a.lanes_shift);
    if (blocks > INT32_MAX / 256) return SR_E_LIMIT;
    embed_kernel<T, O, N><<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(a);
    SR_HIP(hipGetLastError());
    return SR_OK;
}

// ---------------------------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------------------------
constexpr uint32_t kNoToken = 0xffffffffu;           // sorts behind every token
constexpr int kZeroRows = 32;                        // of the table, a workgroup

struct EmbedGradArgs {
    const void *d_out;
    void *d_table;
    const int32_t *tokens;
    int64_t ld_d_out, ld_d_table;
    uint32_t *sorted;                // [n] tokens in order, those outside the vocabulary behind them as kNoToken
    int32_t *places;                 // [n] and where they came from
    float *parts;                    // [chunks][2][width]: sums of the token that comes in from the chunk before, and of the one that goes on
    int n, vocab, width, chunk, chunks, slices, sum_blocks;
    int accumulate;
    float scale;
};

__device__ __forceinline__ uint32_t key_of(int token, int vocab) { return (unsigned)token < (unsigned)vocab ? (uint32_t)token : kNoToken; }

// 64 places a workgroup; each wavefront compares them with a sixteenth of the list, which comes through scalar loads
__global__ __launch_bounds__(1024) void rank_kernel(EmbedGradArgs a) {
    __shared__ int s_rank[16][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int first = (int)blockIdx.x * 64, i = first + lane;
    const uint32_t key = i < a.n ? key_of(a.tokens[i], a.vocab) : kNoToken;
    const int each = (a.n + 15) / 16, from = min(wave * each, a.n), to = min(from + each, a.n);
    int rank = 0;
    // before the workgroup's places: as many as are not greater; among them: by place; behind them: as many as are less
    int j = from;
    for (const int end = min(to, first); j < end; ++j) rank += key_of(read_uniform(a.tokens + j), a.vocab) <= key;
    for (const int end = min(to, first + 64); j < end; ++j) {
        const uint32_t other = key_of(read_uniform(a.tokens + j), a.vocab);
        rank += other < key || (other == key && j < i);
    }
    for (; j < to; ++j) rank += key_of(read_uniform(a.tokens + j), a.vocab) < key;
    s_rank[wave][lane] = rank;
    __syncthreads();
    if (wave != 0 || i >= a.n) return;
    for (int w = 1; w < 16; ++w) rank += s_rank[w][lane];
    a.sorted[rank] = key;
    a.places[rank] = i;
}

// First place of the sorted list whose token is not below `token`; the wavefront asks at 64 places at a time
__device__ __forceinline__ int first_at_least(const uint32_t *sorted, int n, uint32_t token, int lane) {
    int lo = 0, len = n;                             // it lies in [lo, lo + len]
    while (len > 0) {
        const int step = (len + 63) / 64, at = lo + lane * step;
        const int below = __popcll(__ballot(at < lo + len && sorted[at] < token));   // the first `below` asked
        if (below == 0) return lo;
        const int last = lo + (below - 1) * step;    // below `token`; the next one asked is not
        len = min(step, lo + len - last) - 1;
        lo = last + 1;
    }
    return lo;
}

template <int N, typename O>
__device__ __forceinline__ void write_row(const EmbedGradArgs &a, uint32_t token, const Span &s, const float *sum) {
    O *row = (O *)a.d_table + token * a.ld_d_table;
    float y[N];
    if (a.accumulate && s.skip < N) {
        Part<O, N> old;
        old.load(row + s.c);
        old.widen(y);
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = fmaf(a.scale, sum[j], y[j]);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = a.scale * sum[j];
    }
    store_span<N>(row, s, y);
}

// The first sum_blocks workgroups add up chunks, a wavefront a chunk and slice of columns; the others write the zeros of a whole table
template <typename T, typename O, int N>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedGradArgs a) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if ((int)blockIdx.x >= a.sum_blocks) {
        __shared__ uint32_t s_named;
        const uint32_t from = (uint32_t)((int)blockIdx.x - a.sum_blocks) * kZeroRows;
        const uint32_t to = min(from + kZeroRows, (uint32_t)a.vocab);
        if (wave == 0) {
            uint32_t named = 0;
            // one token after the other: the first that is not below the next one
            for (uint32_t next = from; next < to;) {
                const int at = first_at_least(a.sorted, a.n, next, lane);
                const uint32_t token = at < a.n ? read_uniform(a.sorted + at) : kNoToken;
                if (token >= to) break;
                named |= 1u << (token - from);
                next = token + 1;
            }
            if (lane == 0) s_named = named;
        }
        __syncthreads();
        const uint32_t named = s_named;
        const float zero[N] = {};
        const int vecs = (a.width + N - 1) / N;
        for (uint32_t r = from; r < to; ++r) {
            if (named >> (r - from) & 1) continue;
            for (int v = threadIdx.x; v < vecs; v += 256) store_span<N>((O *)a.d_table + r * a.ld_d_table, span_of<N>(v, a.width), zero);
        }
        return;
    }
    const int unit = (int)blockIdx.x * 4 + wave, k = unit / a.slices;
    if (k >= a.chunks) return;
    const Span s = span_of<N>((unit - k * a.slices) * 64 + lane, a.width);
    const int from = k * a.chunk, to = min(from + a.chunk, a.n);
    const uint32_t before = from > 0 ? read_uniform(a.sorted + from - 1) : kNoToken, behind = to < a.n ? read_uniform(a.sorted + to) : kNoToken;
    uint32_t token = read_uniform(a.sorted + from);
    if (token == kNoToken) return;
    bool comes_in = from > 0 && before == token;
    float sum[N];
#pragma unroll
    for (int j = 0; j < N; ++j) sum[j] = 0.f;
    for (int e0 = from; e0 < to; e0 += 64) {
        const int e = min(e0 + lane, to - 1);
        const uint32_t key = a.sorted[e];
        const int place = a.places[e];
        const int count = __popcll(__ballot(e0 + lane < to && key != kNoToken));
        for (int g = 0; g < count; g += 8) {
            Part<T, N> x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                x[u].load((const T *)a.d_out + __builtin_amdgcn_readlane(place, min(g + u, count - 1)) * a.ld_d_out + s.c);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (g + u >= count) break;
                const uint32_t t = __builtin_amdgcn_readlane(key, g + u);
                if (t != token) {
                    if (comes_in) store_span<N>(a.parts + (size_t)(2 * k) * a.width, s, sum);
                    else write_row<N, O>(a, token, s, sum);
                    comes_in = false;
                    token = t;
#pragma unroll
                    for (int j = 0; j < N; ++j) sum[j] = 0.f;
                }
                float y[N];
                x[u].widen(y);
#pragma unroll
                for (int j = 0; j < N; ++j) sum[j] += y[j];
            }
        }
        if (count < 64) break;
    }
    const bool goes_on = behind == token;
    if (comes_in) store_span<N>(a.parts + (size_t)(2 * k) * a.width, s, sum);
    else if (goes_on) store_span<N>(a.parts + (size_t)(2 * k + 1) * a.width, s, sum);
    else write_row<N, O>(a, token, s, sum);
}

// Tokens that reach over the ends of chunks: the workgroup of the chunk that one begins in adds up its parts, each wavefront a run of them
template <typename O, int N>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedGradArgs a) {
    __shared__ float s_sum[3][64][N];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int k = (int)blockIdx.x / a.slices, slice = (int)blockIdx.x - k * a.slices;
    const int from = k * a.chunk, to = from + a.chunk;               // not the last chunk: to < n
    const uint32_t token = read_uniform(a.sorted + to);
    if (token == kNoToken || read_uniform(a.sorted + to - 1) != token) return;
    if (from > 0 && read_uniform(a.sorted + from) == token && read_uniform(a.sorted + from - 1) == token) return;
    // chunks behind this one that begin with the token
    int more = 0;
    for (;;) {
        const int next = k + 1 + more + lane;
        const uint64_t same = __ballot(next < a.chunks && a.sorted[min(next, a.chunks - 1) * a.chunk] == token);
        const int run = ~same ? __ffsll((unsigned long long)~same) - 1 : 64;
        more += run;
        if (run < 64) break;
    }
    const Span s = span_of<N>(slice * 64 + lane, a.width);
    // parts 0 .. more: this chunk's second, the first of those behind it
    const int each = (more + 4) / 4, begin = min(wave * each, more + 1), end = min(begin + each, more + 1);
    float sum[N];
#pragma unroll
    for (int j = 0; j < N; ++j) sum[j] = 0.f;
    for (int p = begin; p < end; p += 4) {
        Part<float, N> x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int q = min(p + u, end - 1);
            x[u].load(a.parts + (size_t)(2 * (k + q) + (q == 0)) * a.width + s.c);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float y[N];
            x[u].widen(y);
#pragma unroll
            for (int j = 0; j < N; ++j) sum[j] += p + u < end ? y[j] : 0.f;
        }
    }
    if (wave) {
#pragma unroll
        for (int j = 0; j < N; ++j) s_sum[wave - 1][lane][j] = sum[j];
    }
    __syncthreads();
    if (wave) return;
    for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] += s_sum[w][lane][j];
    write_row<N, O>(a, token, s, sum);
}

template <typename T, typename O, int N>
int launch_embed_grad(EmbedGradArgs a, hipStream_t stream) {
    if (a.n > 0) {
        rank_kernel<<<dim3(ceil_div(a.n, 64)), dim3(1024), 0, stream>>>(a);
        SR_HIP(hipGetLastError());
    }
    a.sum_blocks = ceil_div(a.chunks * a.slices, 4);
    const int zero_blocks = a.accumulate ? 0 : (int)(((int64_t)a.vocab + kZeroRows - 1) / kZeroRows);
    if (a.sum_blocks + zero_blocks == 0) return SR_OK;
    embed_sum_kernel<T, O, N><<<dim3((unsigned)a.sum_blocks + (unsigned)zero_blocks), dim3(256), 0, stream>>>(a);
    SR_HIP(hipGetLastError());
    if (a.chunks > 1) {
        embed_join_kernel<O, N><<<dim3((unsigned)((a.chunks - 1) * a.slices)), dim3(256), 0, stream>>>(a);
        SR_HIP(hipGetLastError());
    }
    return SR_OK;
}

int embed_grad(const sr_rows *d_out, const int32_t *tokens, int n, float scale, const sr_rows *d_table, int vocab, int width, int accumulate,
               void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!d_out || !d_table || n < 0 || vocab < 1 || width < 1 || !std::isfinite(scale)) return SR_E_ARG;
    if (d_out->dtype < SR_F32 || d_out->dtype > SR_F16 || (d_table->dtype != d_out->dtype && d_table->dtype != SR_F32)) return SR_E_ARG;
    if (n > kMostTokens || width > kMostEmbedWidth) return SR_E_LIMIT;
    if (!rows_fit(*d_table, width, SR_F16) || (n > 0 && (!rows_fit(*d_out, width, SR_F16) || !tokens || (uintptr_t)tokens % 4))) return SR_E_ARG;
    if (n > 0 && d_table->data == d_out->data) return SR_E_ARG;
    if (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < SR_EMBED_GRAD_WORKSPACE(n, width)) return SR_E_ARG;
    if (!accumulate && (int64_t)vocab / kZeroRows + 1 > INT32_MAX / 512) return SR_E_LIMIT;
    const EmbedGradPlan p = embed_grad_plan(n, width, d_out->dtype == SR_F32 || d_table->dtype == SR_F32);
    if ((int64_t)p.chunks * p.slices > INT32_MAX / 512) return SR_E_LIMIT;
    EmbedGradArgs a{};
    a.d_out = d_out->data;
    a.ld_d_out = d_out->ld;
    a.d_table = d_table->data;
    a.ld_d_table = d_table->ld;
    a.tokens = tokens;
    a.sorted = (uint32_t *)workspace;
    a.places = (int32_t *)workspace + n;
    a.parts = (float *)((char *)workspace + round_up(8 * n, 16));
    a.n = n;
    a.vocab = vocab;
    a.width = width;
    a.chunk = p.chunk;
    a.chunks = p.chunks;
    a.slices = p.slices;
    a.accumulate = accumulate != 0;
    a.scale = scale;
    return with_row_types(d_out->dtype, d_table->dtype, [&](auto *t, auto *o) -> int {
        typedef std::remove_pointer_t<decltype(t)> T;
        typedef std::remove_pointer_t<decltype(o)> O;
        constexpr int N = sizeof(O) == 4 ? 4 : 8;
        return p.per_vec == 1 ? launch_embed_grad<T, O, 1>(a, stream) : launch_embed_grad<T, O, N>(a, stream);
    });
}

}  // namespace
}  // namespace sr

extern "C" int sr_embed(const sr_rows *table, int vocab, int width, const int32_t *tokens, int n, float scale, const sr_rows *out,
                        void *stream) {
    using namespace sr;
    if (!table || !out || n < 0 || vocab < 1 || width < 1 || !std::isfinite(scale)) return SR_E_ARG;
    if (table->dtype < SR_F32 || table->dtype > SR_F16 || (out->dtype != table->dtype && out->dtype != SR_F32)) return SR_E_ARG;
    if (width > kMostEmbedWidth) return SR_E_LIMIT;
    if (!rows_fit(*table, width, SR_F16)) return SR_E_ARG;
    if (n == 0) return SR_OK;
    if (!rows_fit(*out, width, SR_F16) || !tokens || (uintptr_t)tokens % 4 || out->data == table->data) return SR_E_ARG;
    EmbedArgs a{table->data, out->data, tokens, table->ld, out->ld, n, vocab, width, 0, FastDiv{}, 0, scale};
    return with_row_types(table->dtype, out->dtype, [&](auto *t, auto *o) -> int {
        typedef std::remove_pointer_t<decltype(t)> T;
        typedef std::remove_pointer_t<decltype(o)> O;
        constexpr int N = sizeof(O) == 4 ? 4 : 8;
        return width < 8 ? launch_embed<T, O, 1>(a, (hipStream_t)stream) : launch_embed<T, O, N>(a, (hipStream_t)stream);
    });
}

extern "C" int sr_embed_grad(const sr_rows *d_out, const int32_t *tokens, int n, float scale, const sr_rows *d_table, int vocab, int width,
                             int accumulate, void *workspace, size_t workspace_bytes, void *stream) {
    return sr::embed_grad(d_out, tokens, n, scale, d_table, vocab, width, accumulate, workspace, workspace_bytes, (hipStream_t)stream);
}
