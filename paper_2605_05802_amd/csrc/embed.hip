// Embedding: rows of a table for a list of tokens, scaled, and the gradient of the table.
//
// out[i] = scale * table[token i]; d_table[v] [+]= scale * sum of d_out[i] over the i whose token is v, in ascending order of i, so that
// the sums are the same bit for bit from call to call.  Tokens outside the vocabulary have a row of zeros and no gradient.
// Memory bounds both; of a whole table's gradient most is zeros to write.
//
// The gradient sorts the tokens and keeps equal ones in order.  The sorted list is cut into chunks of equal length whatever
// tokens they hold, so that a token of half the batch is as well spread as any: a wavefront adds up a chunk's rows, 64 vectors of columns, and
// writes the sums of the tokens that lie in its chunk alone.  Sums of tokens that reach over an end are joined in LDS by the workgroup that has
// kSpanChunks chunks next to each other, and those that reach over its ends by a second kernel, by way of the workspace.
//
// 4096 tokens into a whole table of 152064 x 3584 bf16: 190 us, of which zeros take 160, the sort 6, sums 18 and 5; 49153 tokens, half of
// them one, into 32011 x 1031 fp32: 83 us, 25 + 53 + 5.
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
    const int32_t *tokens;           // null: a whole table of zeros
    int64_t ld_table, ld_out;
    int n, vocab, width, parts;      // parts: wavefronts of a row
    FastDiv by_parts;
    int lanes_shift;                 // log2 of the threads of a row of at most 32 vectors
    float scale;
};

// Rows of at most 32 vectors, several to a wavefront
template <typename T, typename O, int N>
__global__ __launch_bounds__(256) void embed_narrow_kernel(EmbedArgs a) {
    const int row = (int)((blockIdx.x << (8 - a.lanes_shift)) + (threadIdx.x >> a.lanes_shift));
    if (row >= a.n) return;
    const Span s = span_of<N>(threadIdx.x & ((1 << a.lanes_shift) - 1), a.width);
    if (s.skip == N) return;
    const int token = a.tokens ? a.tokens[row] : -1;
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

// A wavefront 64 vectors of a row: its token comes once, through a scalar load.  65536 rows of 3584 bf16: 171 us, as with two, four and eight
// vectors a lane; 190 with a workgroup for 256 vectors, whose second one is three quarters full.
template <typename T, typename O, int N>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a) {
    const int lane = threadIdx.x & 63, unit = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
    const int row = quotient(unit, a.by_parts);
    if (row >= a.n) return;
    const Span s = span_of<N>((unit - row * a.parts) * 64 + lane, a.width);
    const int token = a.tokens ? read_uniform(a.tokens + row) : -1;
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
    if (vecs <= 32) {
        a.lanes_shift = 0;
        while ((1 << a.lanes_shift) < vecs) ++a.lanes_shift;
        const int64_t blocks = ((int64_t)a.n + (256 >> a.lanes_shift) - 1) >> (8 - a.lanes_shift);
        if (blocks > INT32_MAX / 256) return SR_E_LIMIT;
        embed_narrow_kernel<T, O, N><<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(a);
        SR_HIP(hipGetLastError());
        return SR_OK;
    }
    if constexpr (N > 1) {                           // rows column by column are narrow
        a.parts = ceil_div(vecs, 64);
        a.by_parts = fast_div(a.parts);
        const int64_t blocks = ((int64_t)a.n * a.parts + 3) / 4;
        if (blocks > INT32_MAX / 256) return SR_E_LIMIT;
        embed_kernel<T, O, N><<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(a);
        SR_HIP(hipGetLastError());
    }
    return SR_OK;
}

// `bytes` of zeros from an address that an element begins at: 16 bytes a thread, 4 KB a workgroup
__global__ __launch_bounds__(256) void zero_kernel(char *p, size_t bytes) {
    const size_t head = min((size_t)(-(uintptr_t)p & 15), bytes), vecs = (bytes - head) / 16, i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i < vecs) *(raw16 *)(p + head + i * 16) = raw16{0u, 0u, 0u, 0u};
    // pairs of bytes on both sides
    const size_t tail = (bytes - head) & 15;
    if (i < (head + tail) / 2) *(uint16_t *)(p + (i < head / 2 ? 2 * i : bytes - tail + 2 * (i - head / 2))) = 0;
}
int launch_zero(void *data, size_t bytes, hipStream_t stream) {
    constexpr size_t kMost = (size_t)1 << 34;        // of a launch: 2^30 threads
    for (char *p = (char *)data; bytes > 0;) {
        const size_t n = bytes < kMost ? bytes : kMost;
        zero_kernel<<<dim3((unsigned)((n + 4095) / 4096)), dim3(256), 0, stream>>>(p, n);
        SR_HIP(hipGetLastError());
        p += n;
        bytes -= n;
    }
    return SR_OK;
}

// ---------------------------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------------------------
constexpr uint32_t kNoToken = 0x80000000u;           // sorts behind every token
constexpr uint32_t kBehindAll = 0xffffffffu;         // and this behind it
constexpr int kOneTile = 8192;                       // tokens that are sorted by comparing all with all

struct EmbedGradArgs {
    const void *d_out;
    void *d_table;
    const int32_t *tokens;
    int64_t ld_d_out, ld_d_table;
    uint32_t *sorted;                // [n] tokens in order, those outside the vocabulary behind them as kNoToken
    int32_t *places;                 // [n] and where they came from
    uint32_t *other_sorted;          // the same between passes of the sort
    int32_t *other_places;
    uint32_t *counts;                // of digits, of every tile
    float *parts;                    // [spans][2][width]: sums of the token that comes in from the span before, and of the one that goes on
    int n, vocab, width, chunk, spans, slices, sum_blocks;
    int zero_rows;                   // of the table, a workgroup that writes zeros
    FastDiv by_vecs;                 // vectors of a row

    int accumulate;
    float scale;
};

__device__ __forceinline__ int round_up_4(int n) { return (n + 3) & ~3; }
__device__ __forceinline__ uint32_t key_of(int token, int vocab) { return (unsigned)token < (unsigned)vocab ? (uint32_t)token : kNoToken; }

// Short lists: the place of every key is the number of those that come before it.  Sixteen places a workgroup; each group of sixteen lanes
// compares them with its share of the list, which lies in LDS.
constexpr int kRankThreads = 512, kRankGroups = kRankThreads / 16;
__global__ __launch_bounds__(kRankThreads) void rank_kernel(EmbedGradArgs a) {
    __shared__ __align__(16) uint32_t s_key[kOneTile + kOneTile / 16];       // four words more after every 64: groups read different banks
    __shared__ int s_rank[kRankThreads / 64][16];
    const int first = (int)blockIdx.x * 16, each = round_up_4((a.n + kRankGroups - 1) / kRankGroups);        // of a group
    auto slot = [](int j) __attribute__((always_inline)) { return j + (j >> 6) * 4; };
    for (int j0 = threadIdx.x; j0 < each * kRankGroups; j0 += kRankThreads * 8) {        // eight loads before the first is waited for
        int token[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) token[u] = a.tokens[min(j0 + kRankThreads * u, a.n - 1)];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int j = j0 + kRankThreads * u;
            if (j < each * kRankGroups) s_key[slot(j)] = j < a.n ? key_of(token[u], a.vocab) : kBehindAll;
        }
    }
    __syncthreads();
    const int i = (int)threadIdx.x & 15, group = (int)threadIdx.x >> 4;
    const uint32_t key = s_key[slot(min(first + i, a.n - 1))];
    int rank = 0;
    // before the workgroup's places: those that are not greater; from there on: those that are less, and of its own the equal ones before
#pragma unroll 4
    for (int j = group * each; j < (group + 1) * each; j += 4) {
        const raw16 other = *(const raw16 *)(s_key + slot(j));
        const uint32_t limit = key + (j < first);
#pragma unroll
        for (int u = 0; u < 4; ++u) rank += other[u] < limit;
    }
    if (group < i) rank += s_key[slot(min(first + group, a.n - 1))] == key;
    rank += __shfl_xor(rank, 16, 64);
    rank += __shfl_xor(rank, 32, 64);
    if ((threadIdx.x & 63) < 16) s_rank[threadIdx.x >> 6][i] = rank;
    __syncthreads();
    if (threadIdx.x >= 16 || first + i >= a.n) return;
    rank = 0;
#pragma unroll
    for (int w = 0; w < kRankThreads / 64; ++w) rank += s_rank[w][i];
    a.sorted[rank] = key;
    a.places[rank] = first + i;
}

// Longer ones: a stable sort by digits, the lowest first.  A workgroup has a tile of kSortTile keys; a pass counts every tile's digits and then
// moves the keys.  49153 tokens below 32011: 25 us in two passes (with 256 threads a tile 31); comparing tiles of 2048 with all of
// themselves and finding every key's place in the other tiles by search took 30, most of it for loads of single words by address.  Up to kOneTile
// tokens rank_kernel is faster (8192: 22 us with the rest of the call, sorted by digits 32; 4096: 6 us by itself).
constexpr int kSortThreads = 512;
constexpr int kSortRounds = kSortTile / kSortThreads, kWaveKeys = kSortTile / (kSortThreads / 64);
struct SortPass {
    const int32_t *tokens;           // of the first pass, else null
    const uint32_t *keys;
    const int32_t *places;
    uint32_t *to_keys;
    int32_t *to_places;
    uint32_t *counts;                // [tiles][2^BITS]
    int n, tiles, vocab, shift, bits, last;
};
// Tokens outside the vocabulary sort as `vocab`, behind all others; the last pass makes kNoToken of it
__device__ __forceinline__ uint32_t sort_key(const SortPass &p, int i) {
    return p.tokens ? min(key_of(p.tokens[i], p.vocab), (uint32_t)p.vocab) : p.keys[i];
}

// BITS: that a digit has at most
template <int BITS>
__global__ __launch_bounds__(kSortThreads) void digit_count_kernel(SortPass p) {
    constexpr int kDigits = 1 << BITS;
    __shared__ uint32_t s_count[kDigits];
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) s_count[d] = 0;
    __syncthreads();
    const int first = (int)blockIdx.x * kSortTile + (int)threadIdx.x;
    uint32_t key[kSortRounds];
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) key[r] = sort_key(p, min(first + r * kSortThreads, p.n - 1));
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
        if (first + r * kSortThreads < p.n) atomicAdd(&s_count[key[r] >> p.shift & ((1u << p.bits) - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) p.counts[(size_t)blockIdx.x * kDigits + d] = s_count[d];
}

template <int BITS>
__global__ __launch_bounds__(kSortThreads) void digit_move_kernel(SortPass p) {
    constexpr int kWaves = kSortThreads / 64, kDigits = 1 << BITS, kEach = kDigits / kSortThreads, kAhead = 16 / kEach;
    static_assert(kEach == 1 || kEach == 4, "digits of a thread, side by side");
    typedef std::conditional_t<kEach == 1, uint32_t, raw16> Counts;
    __shared__ uint32_t s_at[kWaves][kDigits];       // counts of a wavefront's keys, then the place of its next one
    __shared__ uint32_t s_sum[kWaves];
    const int tile = (int)blockIdx.x, wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63;
    const int first = tile * kSortTile + wave * kWaveKeys + lane;
    uint32_t key[kSortRounds];
    int place[kSortRounds];
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const int i = first + r * 64, at = min(i, p.n - 1);
        key[r] = sort_key(p, at);
        place[r] = p.tokens ? at : p.places[at];
    }
    // of each of the thread's digits: how many there are, and in the tiles before
    Counts all = {}, before = {};
    const Counts *counts = (const Counts *)p.counts + threadIdx.x;
    for (int t = 0; t < p.tiles; t += kAhead) {
        Counts c[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) c[u] = counts[(size_t)min(t + u, p.tiles - 1) * kSortThreads];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            all += c[u] * (uint32_t)(t + u < p.tiles);
            before += c[u] * (uint32_t)(t + u < tile);
        }
    }
    const auto of = [](const Counts &c, int q) __attribute__((always_inline)) -> uint32_t {
        if constexpr (kEach == 1) return c;
        else return c[q];
    };
    for (int i = threadIdx.x; i < kWaves * kDigits; i += kSortThreads) (&s_at[0][0])[i] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
        if (first + r * 64 < p.n) atomicAdd(&s_at[wave][key[r] >> p.shift & ((1u << p.bits) - 1)], 1u);
    // keys of smaller digits
    uint32_t own = 0;
#pragma unroll
    for (int q = 0; q < kEach; ++q) own += of(all, q);
    uint32_t sum = own;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t y = __shfl_up(sum, off, 64);
        if (lane >= off) sum += y;
    }
    if (lane == 63) s_sum[wave] = sum;
    __syncthreads();
    uint32_t base = sum - own;
    for (int w = 0; w < wave; ++w) base += s_sum[w];
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
        uint32_t at = base + of(before, q);
        base += of(all, q);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            uint32_t &to = s_at[w][threadIdx.x * kEach + q];
            const uint32_t c = to;
            to = at;
            at += c;
        }
    }
    __syncthreads();
    // 64 keys after the other: those of a digit among them in order, by comparing digits bit by bit.  (Counted so as well, instead of by atomics, the
    // whole takes 3 to 5 us longer with even tokens and as long with half of them one.)
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const bool here = first + r * 64 < p.n;
        const uint32_t digit = key[r] >> p.shift & ((1u << p.bits) - 1);
        uint64_t same = __ballot(here);
        for (int b = 0; b < p.bits; ++b) {
            const uint64_t set = __ballot(digit >> b & 1);
            same &= digit >> b & 1 ? set : ~set;
        }
        const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
        const uint32_t to = s_at[wave][digit] + rank;
        wave_sync();                                 // all lanes have their place, and the first of a digit moves it on for the next round
        if (here && rank == 0) s_at[wave][digit] = to + __popcll(same);
        wave_sync();
        if (here) {
            p.to_keys[to] = p.last && key[r] == (uint32_t)p.vocab ? kNoToken : key[r];
            p.to_places[to] = place[r];
        }
    }
}

int launch_sort(const EmbedGradArgs &a, hipStream_t stream) {
    if (a.n <= kOneTile) {
        rank_kernel<<<dim3(ceil_div(a.n, 16)), dim3(kRankThreads), 0, stream>>>(a);
        SR_HIP(hipGetLastError());
        return SR_OK;
    }
    // digits of nine bits, and of eleven where those save a pass: a vocabulary below 2048 takes one, of 2^18 to 2^22 two (9000 tokens below 1024: 19.5 us
    // with the rest of the call, in two passes 24.6)
    const int bits = 32 - __builtin_clz((unsigned)a.vocab);
    const bool eleven = ceil_div(bits, kMostDigitBits) < ceil_div(bits, 9);
    const int passes = ceil_div(bits, eleven ? kMostDigitBits : 9), each = ceil_div(bits, passes);
    SortPass p{a.tokens, nullptr, nullptr, nullptr, nullptr, a.counts, a.n, ceil_div(a.n, kSortTile), a.vocab, 0, each, 0};
    for (int k = 0; k < passes; ++k) {
        const bool end = (passes - 1 - k) % 2 == 0;              // the last pass leaves the list where it is read
        p.to_keys = end ? a.sorted : a.other_sorted;
        p.to_places = end ? a.places : a.other_places;
        p.shift = k * each;
        p.last = k + 1 == passes;
        if (eleven) digit_count_kernel<11><<<dim3(p.tiles), dim3(kSortThreads), 0, stream>>>(p);
        else digit_count_kernel<9><<<dim3(p.tiles), dim3(kSortThreads), 0, stream>>>(p);
        SR_HIP(hipGetLastError());
        if (eleven) digit_move_kernel<11><<<dim3(p.tiles), dim3(kSortThreads), 0, stream>>>(p);
        else digit_move_kernel<9><<<dim3(p.tiles), dim3(kSortThreads), 0, stream>>>(p);
        SR_HIP(hipGetLastError());
        p.tokens = nullptr;
        p.keys = p.to_keys;
        p.places = p.to_places;
    }
    return SR_OK;
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

// The first sum_blocks workgroups add up spans of chunks, a wavefront a chunk and slice of columns; the others write the zeros of a whole table
template <typename T, typename O, int N>
__global__ __launch_bounds__(64 * kSpanChunks) void embed_sum_kernel(EmbedGradArgs a) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if ((int)blockIdx.x >= a.sum_blocks) {
        __shared__ int s_bound[2];
        __shared__ uint8_t s_named[kMostZeroRows];
        const uint32_t from = ((uint32_t)blockIdx.x - (uint32_t)a.sum_blocks) * (uint32_t)a.zero_rows;
        const int rows = (int)min((uint32_t)a.zero_rows, (uint32_t)a.vocab - from);
        // the part of the list with these rows, and each of them in it
        if (wave < 2) {
            const int at = first_at_least(a.sorted, a.n, from + (wave ? rows : 0), lane);
            if (lane == 0) s_bound[wave] = at;
        }
        __syncthreads();
        const int end = s_bound[1];
        if ((int)threadIdx.x < rows) {
            int lo = s_bound[0], hi = end;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (a.sorted[mid] < from + threadIdx.x) lo = mid + 1;
                else hi = mid;
            }
            s_named[threadIdx.x] = lo < end && a.sorted[lo] == from + threadIdx.x;
        }
        __syncthreads();
        const float zero[N] = {};
        const int vecs = (a.width + N - 1) / N;
        for (int i = threadIdx.x; i < rows * vecs; i += 64 * kSpanChunks) {
            const int r = quotient(i, a.by_vecs);
            if (!s_named[r]) store_span<N>((O *)a.d_table + (from + r) * a.ld_d_table, span_of<N>(i - r * vecs, a.width), zero);
        }
        return;
    }
    __shared__ float s_sum[kSpanChunks][2][N][64];
    __shared__ uint32_t s_token[kSpanChunks];
    __shared__ int s_kind[kSpanChunks];
    // the slices of a span to one XCD, one soon after the other: they share lines where rows do not begin with one (rows
    // of 1031 halves: 104 MB read instead of 130)
    const int octet = (int)blockIdx.x / (8 * a.slices), rest = (int)blockIdx.x - octet * 8 * a.slices, slice = rest >> 3, span = octet * 8 + (rest & 7);
    if (span >= a.spans) return;
    const Span s = span_of<N>(slice * 64 + lane, a.width);
    const int from = (span * kSpanChunks + wave) * a.chunk, to = min(from + a.chunk, a.n);
    // what becomes of the chunk's first and last sum: kHead, it comes in from before; kTail, a later one goes on behind the chunk;
    // kThrough, the one that comes in goes on
    enum { kHead = 1, kTail = 2, kThrough = 4 };
    int kind = 0;
    uint32_t token = from < to ? read_uniform(a.sorted + from) : kNoToken;
    if (token != kNoToken) {
        const uint32_t before = from > 0 ? read_uniform(a.sorted + from - 1) : kNoToken, behind = to < a.n ? read_uniform(a.sorted + to) : kNoToken;
        bool comes_in = before == token;
        float sum[N];
        auto keep = [&](int which) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < N; ++j) s_sum[wave][which][j][lane] = sum[j];
        };
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
                        if (comes_in) {
                            keep(0);
                            kind = kHead;
                        } else write_row<N, O>(a, token, s, sum);
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
        if (comes_in) {
            keep(0);
            kind = goes_on ? kHead | kThrough : kHead;
        } else if (goes_on) {
            keep(1);
            kind |= kTail;
        } else write_row<N, O>(a, token, s, sum);
    }
    if (lane == 0) {
        s_kind[wave] = kind;
        s_token[wave] = token;                       // of a tail
    }
    __syncthreads();
    if (wave) return;
    // the sums that reach over the ends of chunks, in order: those of one span end here
    float open[N];
    bool outside = false, any = false;
    uint32_t open_token = kNoToken;
    float *parts = a.parts + (size_t)(2 * span) * a.width;
    for (int w = 0; w < kSpanChunks; ++w) {
        const int k = __builtin_amdgcn_readfirstlane(s_kind[w]);
        if (k & kHead) {
            if (w == 0) outside = true;
#pragma unroll
            for (int j = 0; j < N; ++j) open[j] = w == 0 ? s_sum[w][0][j][lane] : open[j] + s_sum[w][0][j][lane];
            any = true;
            if (!(k & kThrough)) {
                if (outside) store_span<N>(parts, s, open);
                else write_row<N, O>(a, open_token, s, open);
                any = outside = false;
            }
        }
        if (k & kTail) {
#pragma unroll
            for (int j = 0; j < N; ++j) open[j] = s_sum[w][1][j][lane];
            any = true;
            open_token = __builtin_amdgcn_readfirstlane(s_token[w]);
        }
    }
    if (any) store_span<N>(outside ? parts : parts + a.width, s, open);
}

// Tokens that reach over the ends of spans: the workgroup of the span that one begins in adds up its parts, each wavefront a run of them
constexpr int kJoinWaves = 8;
template <typename O, int N>
__global__ __launch_bounds__(64 * kJoinWaves) void embed_join_kernel(EmbedGradArgs a) {
    __shared__ float s_sum[kJoinWaves][N][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int k = (int)blockIdx.x / a.slices, slice = (int)blockIdx.x - k * a.slices;
    const int length = kSpanChunks * a.chunk, from = k * length, to = from + length;         // not the last span: to < n
    // asked for together: most workgroups end here
    const uint32_t token = read_uniform(a.sorted + to), last = read_uniform(a.sorted + to - 1), start = read_uniform(a.sorted + from);
    const uint32_t before = read_uniform(a.sorted + max(from - 1, 0));
    if ((token == kNoToken) | (last != token) | ((from > 0) & (start == token) & (before == token))) return;
    // spans behind this one that begin with the token
    int more = 0;
    for (;;) {
        const int next = k + 1 + more + lane;
        const uint64_t same = __ballot(next < a.spans && a.sorted[min(next, a.spans - 1) * length] == token);
        const int run = ~same ? __ffsll((unsigned long long)~same) - 1 : 64;
        more += run;
        if (run < 64) break;
    }
    const Span s = span_of<N>(slice * 64 + lane, a.width);
    // parts 0 .. more: this span's second, the first of those behind it
    const int each = (more + kJoinWaves) / kJoinWaves, begin = min(wave * each, more + 1), end = min(begin + each, more + 1);
    float sum[N];
#pragma unroll
    for (int j = 0; j < N; ++j) sum[j] = 0.f;
    for (int p = begin; p < end; p += 16) {
        Part<float, N> x[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const int q = min(p + u, end - 1);
            x[u].load(a.parts + (size_t)(2 * (k + q) + (q == 0)) * a.width + s.c);
        }
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            float y[N];
            x[u].widen(y);
#pragma unroll
            for (int j = 0; j < N; ++j) sum[j] += p + u < end ? y[j] : 0.f;
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) s_sum[wave][j][lane] = sum[j];
    __syncthreads();
    if (wave) return;
    const int used = min(kJoinWaves, (more + each) / each);
    for (int w = 1; w < used; ++w)
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] += s_sum[w][j][lane];
    write_row<N, O>(a, token, s, sum);
}

// Few tokens and a small table: a workgroup has sixteen rows of the table, looks for them in the whole list and adds up what it finds,
// a wavefront a row; rows with more than kFewTogether places are shared by all.  One launch instead of three: 6.6 us instead of 12.4
// for 256 tokens into 1024 x 256 fp32, of which the call itself is most.
constexpr int kFewTokens = 1024, kFewTogether = 32;
template <typename T, typename O, int N>
__global__ __launch_bounds__(1024) void embed_few_kernel(EmbedGradArgs a) {
    __shared__ float s_sum[16][N][64];
    __shared__ uint16_t s_place[16][kFewTokens];
    __shared__ int s_count[16][16];                  // [wavefront][row]
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, i = threadIdx.x;
    const int block = (int)blockIdx.x / a.slices, slice = (int)blockIdx.x - block * a.slices;
    const uint32_t first = (uint32_t)block * 16;
    const uint32_t key = i < a.n ? key_of(a.tokens[i], a.vocab) : kNoToken, row = key - first;
    int before = 0, mine = 0;                        // of the same row in this wavefront; of row `lane`
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const uint64_t same = __ballot(row == (uint32_t)r);
        if (row == (uint32_t)r) before = __popcll(same & (((uint64_t)1 << lane) - 1));
        if (lane == r) mine = __popcll(same);
    }
    if (lane < 16) s_count[wave][lane] = mine;
    __syncthreads();
    if (row < 16) {
        for (int w = 0; w < wave; ++w) before += s_count[w][row];
        s_place[row][before] = (uint16_t)i;
    }
    // of every row, in lane r
    int count = 0;
    for (int w = 0; w < 16; ++w) count += s_count[w][lane & 15];
    __syncthreads();

    const Span s = span_of<N>(slice * 64 + lane, a.width);
    float sum[N];
    auto add_up = [&](int r, int from, int to) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] = 0.f;
        for (int p = from; p < to; p += 8) {
            Part<T, N> x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                x[u].load((const T *)a.d_out + __builtin_amdgcn_readfirstlane((int)s_place[r][min(p + u, to - 1)]) * a.ld_d_out + s.c);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (p + u >= to) break;
                float y[N];
                x[u].widen(y);
#pragma unroll
                for (int j = 0; j < N; ++j) sum[j] += y[j];
            }
        }
    };
    const int own = __builtin_amdgcn_readlane(count, wave);
    if (own <= kFewTogether && first + wave < (uint32_t)a.vocab) {
        if (own > 0) {
            add_up(wave, 0, own);
            write_row<N, O>(a, first + wave, s, sum);
        } else if (!a.accumulate) {
            const float zero[N] = {};
            store_span<N>((O *)a.d_table + (first + wave) * a.ld_d_table, s, zero);
        }
    }
    for (int r = 0; r < 16; ++r) {
        const int n = __builtin_amdgcn_readlane(count, r);
        if (n <= kFewTogether) continue;             // the same for all wavefronts
        const int each = (n + 15) / 16, from = min(wave * each, n);
        add_up(r, from, min(from + each, n));
#pragma unroll
        for (int j = 0; j < N; ++j) s_sum[wave][j][lane] = sum[j];
        __syncthreads();
        if (wave == 0) {
            for (int w = 1; w < (n + each - 1) / each; ++w)
#pragma unroll
                for (int j = 0; j < N; ++j) sum[j] += s_sum[w][j][lane];
            write_row<N, O>(a, first + r, s, sum);
        }
        __syncthreads();
    }
}

template <typename T, typename O, int N>
int launch_embed_grad(EmbedGradArgs a, hipStream_t stream) {
    if (a.n <= kFewTokens && embed_few(a.vocab, a.slices)) {
        if (a.n == 0 && a.accumulate) return SR_OK;
        embed_few_kernel<T, O, N><<<dim3(ceil_div(a.vocab, 16) * a.slices), dim3(1024), 0, stream>>>(a);
        SR_HIP(hipGetLastError());
        return SR_OK;
    }
    // Few of the rows are named: zeros everywhere first, and the sums over them, because zeros go out fastest by workgroups that write 4 KB each in
    // the order of the memory and ask nothing (1.09 GB in 159 us; wavefronts of 7 KB, whose rows have to be looked for, 198)
    const bool zeros_first = !a.accumulate && zeros_go_first(a.n, a.vocab, a.width * (int64_t)sizeof(O));
    if (zeros_first && a.ld_d_table == a.width) {
        SR_TRY(launch_zero(a.d_table, (size_t)a.vocab * a.width * sizeof(O), stream));
    } else if (zeros_first) {
        const EmbedArgs zeros{nullptr, a.d_table, nullptr, 0, a.ld_d_table, a.vocab, 0, a.width, 0, FastDiv{}, 0, 0.f};
        SR_TRY((launch_embed<O, O, N>(zeros, stream)));
    }
    if (a.n > 0) SR_TRY(launch_sort(a, stream));
    a.sum_blocks = round_up(a.spans, 8) * a.slices;
    a.by_vecs = fast_div(ceil_div(a.width, N));
    const int zero_blocks = a.accumulate || zeros_first ? 0 : ceil_div(a.vocab, a.zero_rows);
    if (a.sum_blocks + zero_blocks == 0) return SR_OK;
    embed_sum_kernel<T, O, N><<<dim3((unsigned)a.sum_blocks + (unsigned)zero_blocks), dim3(64 * kSpanChunks), 0, stream>>>(a);
    SR_HIP(hipGetLastError());
    if (a.spans > 1) {
        embed_join_kernel<O, N><<<dim3((unsigned)((a.spans - 1) * a.slices)), dim3(64 * kJoinWaves), 0, stream>>>(a);
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
    const EmbedGradPlan p = embed_grad_plan(n, width, d_out->dtype == SR_F32 || d_table->dtype == SR_F32, elem_bytes(d_table->dtype));
    if ((int64_t)p.spans * p.slices > INT32_MAX / 1024 || (!accumulate && vocab / p.zero_rows > INT32_MAX / 1024)) return SR_E_LIMIT;
    EmbedGradArgs a{};
    a.d_out = d_out->data;
    a.ld_d_out = d_out->ld;
    a.d_table = d_table->data;
    a.ld_d_table = d_table->ld;
    a.tokens = tokens;
    const EmbedGradRoom room = embed_grad_room(n, width, p);
    char *const at = (char *)workspace;
    a.sorted = (uint32_t *)at;
    a.places = (int32_t *)(at + room.places);
    a.other_sorted = (uint32_t *)(at + room.other_sorted);
    a.other_places = (int32_t *)(at + room.other_places);
    a.counts = (uint32_t *)(at + room.counts);
    a.parts = (float *)(at + room.parts);
    a.n = n;
    a.vocab = vocab;
    a.width = width;
    a.chunk = p.chunk;
    a.spans = p.spans;
    a.slices = p.slices;
    a.zero_rows = p.zero_rows;
    a.accumulate = accumulate != 0;
    a.scale = scale;
    return with_row_types(d_out->dtype, d_table->dtype, [&](auto *t, auto *o) -> int {
        typedef std::remove_pointer_t<decltype(t)> T;
        typedef std::remove_pointer_t<decltype(o)> O;
        constexpr int N = sizeof(O) == 4 ? 4 : 8;    // 8 for 16-bit rows into fp32 as well: 49153 tokens of 1031 98 us, with 4 87
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
    const EmbedArgs a{table->data, out->data, tokens, table->ld, out->ld, n, vocab, width, 0, FastDiv{}, 0, scale};
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
