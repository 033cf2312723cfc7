// Global 2-norm of a list of gradient tensors, and the list scaled down to a largest norm.
//
// norm = |scale| sqrt(sum g^2), out = scale * min(1, max_norm / norm) * g.  Memory bounds it.  Two passes over the data, because no
// element may be written before the last one has been read: every gradient is read twice and written once, unless the caches
// still hold it.  The first pass reads the last kKeepBytes with default loads, which leave them in the memory-side cache, and what
// comes before with the non-temporal hint, which is faster (2 GB of bf16: 296 us, 6.8 TB/s; all with default loads 321) but leaves nothing
// behind (the second pass over 0.47 GB of bf16 into fp32 took 265 us where all had been read so, and 233 where none had).
// 2 GB of bf16 into bf16: 296 + 636 us (6.4 TB/s) of 941 a call; the list of a small model: two launches, which cost more than their work.
//
// A list travels in the kernel arguments, kListTensors tensors a launch: no copy to the device, nothing kept between calls, and a
// captured launch holds its own list.  A planned list lies on the device, of any length, for one launch a pass: 339 tensors of 20 000
// elements on average take 17 us, 24 in the arguments of two.  A chunk of kChunk elements is a workgroup's step; its tensor is found by
// comparing 64 first chunks at a time.
#include <cmath>
#include <cstdlib>

#include "row_vectors.h"

namespace sr {
namespace {

constexpr int kListTensors = 184;      // with the hidden ones 4 KB of kernel arguments
constexpr int kLdsTensors = 512;       // of a list that square_sum_kernel copies to LDS
constexpr int kChunk = 8192;           // elements
constexpr int kNormThreads = 256;
constexpr int kMostBlocks = 1024;      // workgroups of a launch
constexpr int64_t kMostChunks = 1 << 23;                   // of a launch: 2^31 threads
constexpr int64_t kMostElements = kMostChunks * kChunk;    // of a tensor
constexpr int kSlots = 2048;           // sums that the workspace holds
constexpr int kMostSummed = 2048;      // chunks whose workgroups each add the slots up
constexpr int64_t kKeepBytes = 256 << 20;
static_assert(kSlots * 8 <= SR_GRAD_NORM_WORKSPACE, "workspace");

// A tensor is an address of 48 bits with, above them, the elements of its last chunk (13 bits, 0 for all of them) and its type.
constexpr int kAddressBits = 48, kTypeShift = 61;
struct TensorList {
    uint64_t data[kListTensors];
    uint64_t out[kListTensors];        // address and type
    uint32_t first[kListTensors + 1];  // chunk at which a tensor begins; behind the last one the number of chunks
    int32_t tensors;
};
static_assert(sizeof(TensorList) + 32 + 256 <= 4096, "kernel arguments");

// The same on the device
struct TensorTable {
    const uint64_t *data, *out;
    const uint32_t *first;
    int32_t tensors;
};

struct Chunk {
    char *data, *out;                  // of the chunk's first element
    int n, type, out_type;
};

// A chunk of tensor t, which begins at chunk `from` and ends before chunk `to` of the launch
__device__ __forceinline__ Chunk chunk_of(uint64_t data, uint64_t out, uint32_t from, uint32_t to, uint32_t chunk) {
    constexpr uint64_t address = ((uint64_t)1 << kAddressBits) - 1;
    const uint32_t at = chunk - from;
    const int rest = (int)(data >> kAddressBits) & (kChunk - 1);
    Chunk c;
    c.n = chunk + 1 == to && rest ? rest : kChunk;
    c.type = (int)(data >> kTypeShift);
    c.out_type = (int)(out >> kTypeShift);
    c.data = (char *)(data & address) + (uint64_t)at * (kChunk * (c.type == SR_F32 ? 4 : 2));
    c.out = (char *)(out & address) + (uint64_t)at * (kChunk * (c.out_type == SR_F32 ? 4 : 2));
    return c;
}

// The workgroup's copy of a list of at most kLdsTensors
struct ListInLds {
    uint64_t data[kLdsTensors];
    uint32_t first[kLdsTensors + 64];  // behind the tensors: no chunk

    template <typename List>
    __device__ __forceinline__ void fill(const List &l) {
        for (int i = threadIdx.x; i < l.tensors; i += kNormThreads) data[i] = l.data[i];
        for (int i = threadIdx.x; i < (l.tensors & ~63) + 64; i += kNormThreads) first[i] = i <= l.tensors ? l.first[i] : 0xffffffffu;
    }
    // Every wavefront for itself: tensors that begin at or before the chunk, 64 compared at a time
    __device__ __forceinline__ Chunk find(int tensors, uint32_t chunk) const {
        int t = -1;
        for (int k = 0; k <= tensors; k += 64) t += __popcll(__ballot(first[k + (threadIdx.x & 63)] <= chunk));
        return chunk_of(data[t], 0, first[t], first[t + 1], chunk);
    }
};
// The same from the kernel's arguments
__device__ __forceinline__ Chunk find_chunk(const TensorList &l, uint32_t chunk) {
    int t = -1;
    for (int k = 0; k < l.tensors; k += 64) {
        const int i = k + (int)(threadIdx.x & 63);
        t += __popcll(__ballot(i < l.tensors && l.first[i] <= chunk));
    }
    t = __builtin_amdgcn_readfirstlane(t);
    return chunk_of(l.data[t], l.out[t], l.first[t], l.first[t + 1], chunk);
}
// ... and from a table: the one of 64 shares of what is left that the chunk lies in, until that is one tensor
__device__ __forceinline__ Chunk find_chunk(const TensorTable &l, uint32_t chunk) {
    int t = 0;
    for (int n = l.tensors; n > 1;) {
        const int step = (n + 63) / 64, i = (int)(threadIdx.x & 63) * step;
        const int past = __popcll(__ballot(i < n && l.first[t + i] <= chunk)) - 1;     // the first one is
        t += past * step;
        n = min(step, n - past * step);
    }
    t = __builtin_amdgcn_readfirstlane(t);
    return chunk_of(read_uniform(l.data + t), read_uniform(l.out + t), read_uniform(l.first + t), read_uniform(l.first + t + 1), chunk);
}
static_assert(kListTensors <= kLdsTensors && kLdsTensors % 64 == 0, "capacity");

// f(vector j of the thread, its element) for the chunk's whole vectors of N elements, j known to the compiler; WHOLE: all are there
template <int N, bool WHOLE, typename F>
__device__ __forceinline__ void each_vector(int n, F &&f) {
#pragma unroll
    for (int j = 0; j < kChunk / (kNormThreads * N); ++j) {
        const int e = (j * kNormThreads + (int)threadIdx.x) * N;
        if (WHOLE || e + N <= n) f(j, e);
    }
}

// KEEP: with default loads, which leave the data in the memory-side cache
template <typename T, bool WHOLE, bool KEEP>
__device__ __forceinline__ double squares_of(const T *p, int n) {
    constexpr int N = Elem<T>::kPerVec;
    raw16 raw[kChunk / (kNormThreads * N)];
    double acc = 0.0;
    // the two forms differ in a hint alone, and the compiler would make one of them that has lost it
    asm volatile("; keep %0" ::"n"((int)KEEP));
    each_vector<N, WHOLE>(n, [&](int j, int e) __attribute__((always_inline)) { raw[j] = KEEP ? load_vec(p + e) : load_vec_once(p + e); });
    asm volatile("; keep %0" ::"n"((int)KEEP));
    if (!WHOLE && (int)threadIdx.x < n % N) {
        const double x = (double)(float)p[n / N * N + threadIdx.x];
        acc = x * x;
    }
    each_vector<N, WHOLE>(n, [&](int j, int) __attribute__((always_inline)) {
        float x[N];
        Elem<T>::widen(raw[j], x);
#pragma unroll
        for (int i = 0; i < N; ++i) acc = fma((double)x[i], (double)x[i], acc);
    });
    return acc;
}
template <typename T>
__device__ __forceinline__ double squares(const T *p, int n, bool keep) {
    if (n != kChunk) return squares_of<T, false, true>(p, n);
    return keep ? squares_of<T, true, true>(p, n) : squares_of<T, true, false>(p, n);
}

// add: the slots hold the sums of an earlier launch of the same call; keep: chunks from here on are read again by scale_kernel
template <typename List>
__global__ __launch_bounds__(kNormThreads) void square_sum_kernel(List l, double *__restrict__ slots, int add, uint32_t keep) {
    __shared__ ListInLds list;
    __shared__ double s[kNormThreads / 64];
    const bool in_lds = l.tensors <= kLdsTensors;
    if (in_lds) list.fill(l);
    __syncthreads();
    const uint32_t chunks = l.first[l.tensors];
    double acc = 0.0;
    for (uint32_t k = blockIdx.x; k < chunks; k += gridDim.x) {
        const Chunk c = in_lds ? list.find(l.tensors, k) : find_chunk(l, k);
        acc += c.type == SR_F32    ? squares((const float *)c.data, c.n, k >= keep)
               : c.type == SR_BF16 ? squares((const __bf16 *)c.data, c.n, k >= keep)
                                   : squares((const f16_t *)c.data, c.n, k >= keep);
    }
    acc = block_sum<kNormThreads / 64>(acc, s);
    if (threadIdx.x == 0) slots[blockIdx.x] = (add ? slots[blockIdx.x] : 0.0) + acc;
}

// The squared norm from the slots, in every thread; s: kNormThreads / 64 + 1 doubles of LDS.  The order of the sum is that of the
// slots' numbers.
__device__ __forceinline__ double sum_slots(const double *__restrict__ slots, int used, double *s) {
    if (used == 1) return slots[0];
    double acc = 0.0;
    for (int i = threadIdx.x; i < used; i += kNormThreads) acc += slots[i];
    acc = block_sum<kNormThreads / 64>(acc, s);
    if (threadIdx.x == 0) s[kNormThreads / 64] = acc;
    __syncthreads();
    return s[kNormThreads / 64];
}

// The sum is left in the first slot
__global__ __launch_bounds__(kNormThreads) void norm_kernel(double *slots, int used, float scale, float *__restrict__ norm) {
    __shared__ double s[kNormThreads / 64 + 1];
    const double sum = used ? sum_slots(slots, used, s) : 0.0;
    if (threadIdx.x != 0) return;
    slots[0] = sum;
    *norm = (float)(fabs((double)scale) * sqrt(sum));
}

// What to multiply by, in two steps: where the whole of it is below the smallest normal number, 2^100 times it, which has all its bits, and
// 2^-100.  Else the second is 1 and changes nothing (one product more an element of a kernel that waits for memory).
struct Factor {
    float first, second;
};
__device__ __forceinline__ Factor factor_of(double x) {
    if (fabs(x) < (double)FLT_MIN) return Factor{(float)(x * 0x1p100), 0x1p-100f};
    return Factor{(float)x, 1.f};
}

// Four elements a thread and step where 16-bit data become single precision, so that whole lines are written at once.
// factor(): what to multiply by, asked for when the loads are under way.
template <typename T, typename U, bool WHOLE, typename F>
__device__ __forceinline__ void scale_some(const T *p, U *q, int n, F &&factor) {
    constexpr bool WIDER = sizeof(U) > sizeof(T);
    constexpr int N = Elem<U>::kPerVec;
    raw16 raw[kChunk / (kNormThreads * N)];
    each_vector<N, WHOLE>(n, [&](int j, int e) __attribute__((always_inline)) {
        if constexpr (WIDER) {
            const raw8 half = load_half_vec_once(p + e);
            raw[j] = raw16{half[0], half[1], 0u, 0u};
        } else {
            raw[j] = load_vec_once(p + e);
        }
    });
    const int rest = n / N * N + (int)threadIdx.x;
    float last = 0.f;
    if (!WHOLE && rest < n) last = (float)p[rest];
    const Factor c = factor();
    if (!WHOLE && rest < n) q[rest] = (U)(last * c.first * c.second);
    each_vector<N, WHOLE>(n, [&](int j, int e) __attribute__((always_inline)) {
        float x[Elem<T>::kPerVec];
        Elem<T>::widen(raw[j], x);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = x[i] * c.first * c.second;
        store_vec_once(q + e, Elem<U>::narrow(x));
    });
}
template <typename T, typename U, typename F>
__device__ __forceinline__ void scale_chunk(const Chunk &k, F &&factor) {
    if (k.n == kChunk) scale_some<T, U, true>((const T *)k.data, (U *)k.out, k.n, factor);
    else scale_some<T, U, false>((const T *)k.data, (U *)k.out, k.n, factor);
}

// One chunk a workgroup, in the order of the list: 2 GB of bf16 in 636 us; where 1024 workgroups took chunks in turn
// it was 732, and this way 657 then.
// chunk0: that of the launch's first workgroup
template <typename List>
__global__ __launch_bounds__(kNormThreads) void scale_kernel(List l, uint32_t chunk0, const double *__restrict__ slots, int used, float scale,
                                                             float max_norm, float *__restrict__ norm_out) {
    __shared__ double s[kNormThreads / 64 + 1];
    const Chunk k = find_chunk(l, chunk0 + blockIdx.x);
    auto factor = [&]() __attribute__((always_inline)) {     // holds barriers: once, by the whole workgroup
        const double norm = fabs((double)scale) * sqrt(sum_slots(slots, used, s));
        const float written = (float)norm;                   // the caller knows this one: infinite beyond FLT_MAX, and then nothing is scaled
        if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = written;
        // a quotient of doubles, rounded once; false for NaN
        return norm > (double)max_norm && written <= FLT_MAX ? factor_of((double)scale * ((double)max_norm / norm)) : Factor{scale, 1.f};
    };
    auto scale_by = [&](auto &&f) __attribute__((always_inline)) {
        switch (k.type * 4 + k.out_type) {
            case SR_F32 * 4 + SR_F32: scale_chunk<float, float>(k, f); break;
            case SR_BF16 * 4 + SR_F32: scale_chunk<__bf16, float>(k, f); break;
            case SR_F16 * 4 + SR_F32: scale_chunk<f16_t, float>(k, f); break;
            case SR_BF16 * 4 + SR_BF16: scale_chunk<__bf16, __bf16>(k, f); break;
            case SR_F16 * 4 + SR_F16: scale_chunk<f16_t, f16_t>(k, f); break;
        }
    };
    if (k.data != k.out) return scale_by(factor);
    const Factor c = factor();                               // in place: nothing is read where nothing changes
    if (c.first != 1.f) scale_by([&]() { return c; });
}

int check_tensor(const sr_tensor &t, bool clip) {
    if (t.n < 0 || t.n > kMostElements || t.dtype < SR_F32 || t.dtype > SR_F16) return SR_E_ARG;
    if (t.n == 0) return SR_OK;
    if (!t.data || (uintptr_t)t.data % (t.dtype == SR_F32 ? 4 : 2) || (uintptr_t)t.data >> kAddressBits) return SR_E_ARG;
    if (!clip || !t.out) return SR_OK;
    if (t.out_dtype != t.dtype && t.out_dtype != SR_F32) return SR_E_ARG;
    if ((uintptr_t)t.out % (t.out_dtype == SR_F32 ? 4 : 2) || (uintptr_t)t.out >> kAddressBits) return SR_E_ARG;
    return t.out == t.data && t.out_dtype != t.dtype ? SR_E_ARG : SR_OK;
}

uint64_t packed_data(const sr_tensor &t) {
    return (uint64_t)(uintptr_t)t.data | (uint64_t)(t.n % kChunk) << kAddressBits | (uint64_t)t.dtype << kTypeShift;
}
uint64_t packed_out(const sr_tensor &t) {
    return (uint64_t)(uintptr_t)(t.out ? t.out : t.data) | (uint64_t)(t.out ? t.out_dtype : t.dtype) << kTypeShift;
}
int64_t tensor_bytes(const sr_tensor &t) { return t.n * (t.dtype == SR_F32 ? 4 : 2); }

// A launch's share of the list: tensors from `at` on; returns where the next share begins.  A launch has at most kMostChunks chunks.
int take(const sr_tensor *tensors, int n_tensors, int at, TensorList *l) {
    l->tensors = 0;
    l->first[0] = 0;
    for (; at < n_tensors && l->tensors < kListTensors; ++at) {
        const sr_tensor &t = tensors[at];
        if (t.n == 0) continue;
        const int64_t chunks = (t.n + kChunk - 1) / kChunk + l->first[l->tensors];
        if (chunks > kMostChunks) break;
        const int i = l->tensors++;
        l->data[i] = packed_data(t);
        l->out[i] = packed_out(t);
        l->first[i + 1] = (uint32_t)chunks;
    }
    return at;
}

int check_norm(float scale, float max_norm, const float *norm, const void *workspace, size_t workspace_bytes) {
    return norm && (uintptr_t)norm % 4 == 0 && workspace && (uintptr_t)workspace % 16 == 0 && workspace_bytes >= SR_GRAD_NORM_WORKSPACE &&
                   std::isfinite(scale) && std::isfinite(max_norm) && max_norm >= 0.f
               ? SR_OK
               : SR_E_ARG;
}

int norm_and_clip(const sr_tensor *tensors, int n_tensors, float scale, float max_norm, bool clip, float *norm, void *workspace,
                  size_t workspace_bytes, hipStream_t stream) {
    if (n_tensors < 0 || (n_tensors > 0 && !tensors)) return SR_E_ARG;
    SR_TRY(check_norm(scale, max_norm, norm, workspace, workspace_bytes));
    int64_t bytes = 0;                                   // of what the next launches read
    for (int i = 0; i < n_tensors; ++i) {
        SR_TRY(check_tensor(tensors[i], clip));
        bytes += tensor_bytes(tensors[i]);
    }
    double *slots = (double *)workspace;
    TensorList l;
    int used = 0;
    int64_t chunks = 0;
    for (int at = 0; at < n_tensors;) {
        const int from = at;
        at = take(tensors, n_tensors, at, &l);
        if (!l.tensors) continue;
        // the chunk from which on at most kKeepBytes of the list are left
        uint32_t keep = 0;
        for (int i = from; i < at; ++i) {
            const int64_t n = tensor_bytes(tensors[i]), before = bytes - kKeepBytes;
            if (before > 0) keep += (uint32_t)(((before < n ? before : n) / (tensors[i].dtype == SR_F32 ? 4 : 2) + kChunk - 1) / kChunk);
            bytes -= n;
        }
        const int blocks = l.first[l.tensors] < kMostBlocks ? (int)l.first[l.tensors] : kMostBlocks;
        const bool fits = used + blocks <= kSlots;       // if not, more than kSlots - kMostBlocks >= kMostBlocks of them are in use
        square_sum_kernel<<<dim3(blocks), dim3(kNormThreads), 0, stream>>>(l, fits ? slots + used : slots, !fits, clip ? keep : UINT32_MAX);
        SR_HIP(hipGetLastError());
        if (fits) used += blocks;
        chunks += l.first[l.tensors];
    }
    // few chunks: the workgroups that scale them add the slots up for themselves, and a launch is saved
    const bool alone = !clip || used == 0 || chunks > kMostSummed;
    if (alone) {
        norm_kernel<<<dim3(1), dim3(kNormThreads), 0, stream>>>(slots, used, scale, norm);
        SR_HIP(hipGetLastError());
        used = 1;
    }
    float *out = alone ? nullptr : norm;
    for (int at = 0; clip && at < n_tensors;) {
        at = take(tensors, n_tensors, at, &l);
        if (!l.tensors) continue;
        scale_kernel<<<dim3(l.first[l.tensors]), dim3(kNormThreads), 0, stream>>>(l, 0u, slots, used, scale, max_norm, out);
        SR_HIP(hipGetLastError());
        out = nullptr;
    }
    return SR_OK;
}

// A planned list's table: packed data, packed outputs, first chunks
TensorTable table_of(const sr_tensor_plan &p) {
    const uint64_t *t = (const uint64_t *)p.table;
    return TensorTable{t, t + p.n_tensors, (const uint32_t *)(t + 2 * (size_t)p.n_tensors), p.n_tensors};
}

int plan_tensors(const sr_tensor *tensors, int n_tensors, void *table, size_t table_bytes, sr_tensor_plan *plan, hipStream_t stream) {
    if (n_tensors < 0 || (n_tensors > 0 && !tensors) || !table || (uintptr_t)table % 16 || !plan) return SR_E_ARG;
    if (table_bytes < SR_TENSOR_TABLE_BYTES(n_tensors)) return SR_E_ARG;
    int64_t bytes = 0, chunks = 0, keep = 0;
    int used = 0;
    for (int i = 0; i < n_tensors; ++i) {
        SR_TRY(check_tensor(tensors[i], true));
        if (tensors[i].n == 0) continue;
        bytes += tensor_bytes(tensors[i]);
        chunks += (tensors[i].n + kChunk - 1) / kChunk;
        ++used;
    }
    if (chunks > INT32_MAX) return SR_E_LIMIT;
    const size_t size = (size_t)20 * used + 4;
    char *host = (char *)malloc(size);
    if (!host) return SR_E_NOMEM;
    uint64_t *data = (uint64_t *)host, *out = data + used;
    uint32_t *first = (uint32_t *)(out + used);
    int at = 0;
    first[0] = 0;
    for (int i = 0; i < n_tensors; ++i) {
        const sr_tensor &t = tensors[i];
        if (t.n == 0) continue;
        data[at] = packed_data(t);
        out[at] = packed_out(t);
        first[at + 1] = first[at] + (uint32_t)((t.n + kChunk - 1) / kChunk);
        const int64_t n = tensor_bytes(t), before = bytes - kKeepBytes;
        if (before > 0) keep += ((before < n ? before : n) / (t.dtype == SR_F32 ? 4 : 2) + kChunk - 1) / kChunk;
        bytes -= n;
        ++at;
    }
    hipError_t e = hipMemcpyAsync(table, host, size, hipMemcpyHostToDevice, stream);
    if (e == hipSuccess) e = hipStreamSynchronize(stream);
    free(host);
    SR_HIP(e);
    *plan = sr_tensor_plan{table, chunks, keep, used, 0};
    return SR_OK;
}

int planned_norm_and_clip(const sr_tensor_plan *plan, float scale, float max_norm, bool clip, float *norm, void *workspace,
                          size_t workspace_bytes, hipStream_t stream) {
    if (!plan || !plan->table || plan->n_tensors < 0 || plan->chunks < plan->n_tensors || plan->chunks > INT32_MAX) return SR_E_ARG;
    SR_TRY(check_norm(scale, max_norm, norm, workspace, workspace_bytes));
    double *slots = (double *)workspace;
    const TensorTable l = table_of(*plan);
    const int64_t chunks = l.tensors ? plan->chunks : 0;
    int used = chunks < kMostBlocks ? (int)chunks : kMostBlocks;
    if (used) {
        square_sum_kernel<<<dim3(used), dim3(kNormThreads), 0, stream>>>(l, slots, 0, clip ? (uint32_t)plan->keep : UINT32_MAX);
        SR_HIP(hipGetLastError());
    }
    const bool alone = !clip || used == 0 || chunks > kMostSummed;
    if (alone) {
        norm_kernel<<<dim3(1), dim3(kNormThreads), 0, stream>>>(slots, used, scale, norm);
        SR_HIP(hipGetLastError());
        used = 1;
    }
    float *out = alone ? nullptr : norm;
    for (int64_t at = 0; clip && at < chunks; at += kMostChunks) {
        const int64_t n = chunks - at < kMostChunks ? chunks - at : kMostChunks;
        scale_kernel<<<dim3((unsigned)n), dim3(kNormThreads), 0, stream>>>(l, (uint32_t)at, slots, used, scale, max_norm, out);
        SR_HIP(hipGetLastError());
        out = nullptr;
    }
    return SR_OK;
}

}  // namespace
}  // namespace sr

extern "C" int sr_grad_norm(const sr_tensor *host_tensors, int n_tensors, float scale, float *norm, void *workspace,
                            size_t workspace_bytes, void *stream) {
    return sr::norm_and_clip(host_tensors, n_tensors, scale, 0.f, false, norm, workspace, workspace_bytes, (hipStream_t)stream);
}

extern "C" int sr_clip_grad_norm(const sr_tensor *host_tensors, int n_tensors, float scale, float max_norm, float *norm,
                                 void *workspace, size_t workspace_bytes, void *stream) {
    return sr::norm_and_clip(host_tensors, n_tensors, scale, max_norm, true, norm, workspace, workspace_bytes, (hipStream_t)stream);
}

extern "C" int sr_plan_tensors(const sr_tensor *host_tensors, int n_tensors, void *table, size_t table_bytes, sr_tensor_plan *host_plan,
                               void *stream) {
    return sr::plan_tensors(host_tensors, n_tensors, table, table_bytes, host_plan, (hipStream_t)stream);
}

extern "C" int sr_planned_grad_norm(const sr_tensor_plan *host_plan, float scale, float *norm, void *workspace, size_t workspace_bytes,
                                    void *stream) {
    return sr::planned_norm_and_clip(host_plan, scale, 0.f, false, norm, workspace, workspace_bytes, (hipStream_t)stream);
}

extern "C" int sr_planned_clip_grad_norm(const sr_tensor_plan *host_plan, float scale, float max_norm, float *norm, void *workspace,
                                         size_t workspace_bytes, void *stream) {
    return sr::planned_norm_and_clip(host_plan, scale, max_norm, true, norm, workspace, workspace_bytes, (hipStream_t)stream);
}
