// Global 2-norm of a list of gradient tensors, and the list scaled down to a largest norm.
//
// norm = |scale| sqrt(sum g^2), out = scale * min(1, max_norm / norm) * g.  Two passes over the data, because no element
// may be written before the last one has been read: what has to move is each gradient read once and written once, and the
// second reading on top wherever the list does not fit the caches.
//
// The list travels in the kernel arguments, kListTensors tensors a launch: no copy to the device, nothing kept between calls, and a
// captured launch holds its own list.  A workgroup takes chunks of kChunk elements in turn and finds a chunk's tensor by
// bisection over the uniform prefix counts.
#include <cmath>

#include "row_vectors.h"

namespace sr {
namespace {

constexpr int kListTensors = 120;      // 3.5 KB of kernel arguments
constexpr int kChunk = 8192;           // elements
constexpr int kNormThreads = 256;
constexpr int kMostBlocks = 2048;      // workgroups of a launch
constexpr int kSlots = SR_GRAD_NORM_WORKSPACE / 8;

struct TensorList {
    const void *data[kListTensors];
    void *out[kListTensors];
    int64_t n[kListTensors];
    uint32_t first[kListTensors + 1];  // chunk at which a tensor begins; behind the last one the number of chunks
    uint8_t dtype[kListTensors], out_dtype[kListTensors];
    int32_t tensors;
};

// tensor of a chunk: the last one that begins at or before it (empty tensors begin where the next one does)
__device__ __forceinline__ int tensor_of(const TensorList &l, uint32_t chunk) {
    int lo = 0, hi = l.tensors;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (l.first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

template <typename T>
__device__ __forceinline__ double squares(const T *p, int64_t at, int64_t n) {
    constexpr int N = Elem<T>::kPerVec;
    const int64_t end = at + kChunk < n ? at + kChunk : n;
    double acc = 0.0;
    for (int64_t e = at + (int64_t)threadIdx.x * N; e < end; e += kNormThreads * N) {
        float x[N];
        load_widened(p, e, n, 0.f, x);
#pragma unroll
        for (int i = 0; i < N; ++i) acc = fma((double)x[i], (double)x[i], acc);
    }
    return acc;
}

// add: the slots hold the sums of an earlier launch of the same call
__global__ __launch_bounds__(kNormThreads) void square_sum_kernel(TensorList l, double *__restrict__ slots, int add) {
    __shared__ double s[kNormThreads / 64];
    const uint32_t chunks = l.first[l.tensors];
    double acc = 0.0;
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int t = tensor_of(l, c);
        const int64_t at = (int64_t)(c - l.first[t]) * kChunk;
        acc += l.dtype[t] == SR_F32    ? squares((const float *)l.data[t], at, l.n[t])
               : l.dtype[t] == SR_BF16 ? squares((const __bf16 *)l.data[t], at, l.n[t])
                                       : squares((const f16_t *)l.data[t], at, l.n[t]);
    }
    acc = block_sum<kNormThreads / 64>(acc, s);
    if (threadIdx.x == 0) slots[blockIdx.x] = (add ? slots[blockIdx.x] : 0.0) + acc;
}

__global__ __launch_bounds__(kNormThreads) void norm_kernel(double *__restrict__ slots, int used, float scale, float *__restrict__ norm) {
    __shared__ double s[kNormThreads / 64];
    double acc = 0.0;
    for (int i = threadIdx.x; i < used; i += kNormThreads) acc += slots[i];
    acc = block_sum<kNormThreads / 64>(acc, s);
    if (threadIdx.x == 0) {
        const double x = fabs((double)scale) * sqrt(acc);
        slots[0] = x;
        *norm = (float)x;
    }
}

template <typename T, typename U>
__device__ __forceinline__ void scale_chunk(const T *p, U *q, int64_t at, int64_t n, float c) {
    constexpr int N = Elem<T>::kPerVec, NU = Elem<U>::kPerVec;
    const int64_t end = at + kChunk < n ? at + kChunk : n;
    for (int64_t e = at + (int64_t)threadIdx.x * N; e < end; e += kNormThreads * N) {
        float x[N];
        load_widened(p, e, n, 0.f, x);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= c;
#pragma unroll
        for (int i = 0; i < N; i += NU) store_narrowed(q, e + i, n, x + i);
    }
}

__global__ __launch_bounds__(kNormThreads) void scale_kernel(TensorList l, const double *__restrict__ slots, float scale, float max_norm) {
    const double norm = slots[0];
    // a quotient of doubles, rounded once; false for NaN
    const float c = norm > (double)max_norm && norm <= DBL_MAX ? (float)((double)scale * ((double)max_norm / norm)) : scale;
    const uint32_t chunks = l.first[l.tensors];
    for (uint32_t k = blockIdx.x; k < chunks; k += gridDim.x) {
        const int t = tensor_of(l, k);
        const int64_t at = (int64_t)(k - l.first[t]) * kChunk, n = l.n[t];
        const void *p = l.data[t];
        void *q = l.out[t];
        if (p == q && c == 1.f) continue;
        switch (l.dtype[t] * 4 + l.out_dtype[t]) {
            case SR_F32 * 4 + SR_F32: scale_chunk((const float *)p, (float *)q, at, n, c); break;
            case SR_BF16 * 4 + SR_F32: scale_chunk((const __bf16 *)p, (float *)q, at, n, c); break;
            case SR_F16 * 4 + SR_F32: scale_chunk((const f16_t *)p, (float *)q, at, n, c); break;
            case SR_BF16 * 4 + SR_BF16: scale_chunk((const __bf16 *)p, (__bf16 *)q, at, n, c); break;
            case SR_F16 * 4 + SR_F16: scale_chunk((const f16_t *)p, (f16_t *)q, at, n, c); break;
        }
    }
}

int check_tensor(const sr_tensor &t, bool clip) {
    if (t.n < 0 || t.n >= (int64_t)1 << 43 || t.dtype < SR_F32 || t.dtype > SR_F16) return SR_E_ARG;
    if (t.n == 0) return SR_OK;
    if (!t.data || (uintptr_t)t.data % (t.dtype == SR_F32 ? 4 : 2)) return SR_E_ARG;
    if (!clip || !t.out) return SR_OK;
    if (t.out_dtype != t.dtype && t.out_dtype != SR_F32) return SR_E_ARG;
    if ((uintptr_t)t.out % (t.out_dtype == SR_F32 ? 4 : 2)) return SR_E_ARG;
    return t.out == t.data && t.out_dtype != t.dtype ? SR_E_ARG : SR_OK;
}

// The next launch's share of the list, from tensor `at` on; returns where the one behind it begins.  The counts of chunks stay
// below 2^31.
int take(const sr_tensor *tensors, int n_tensors, int at, TensorList *l) {
    l->tensors = 0;
    l->first[0] = 0;
    for (; at < n_tensors && l->tensors < kListTensors; ++at) {
        const sr_tensor &t = tensors[at];
        if (t.n == 0) continue;
        const int64_t chunks = (t.n + kChunk - 1) / kChunk + l->first[l->tensors];
        if (chunks > INT32_MAX) break;
        const int i = l->tensors++;
        l->data[i] = t.data;
        l->out[i] = t.out ? t.out : t.data;
        l->n[i] = t.n;
        l->dtype[i] = (uint8_t)t.dtype;
        l->out_dtype[i] = (uint8_t)(t.out ? t.out_dtype : t.dtype);
        l->first[i + 1] = (uint32_t)chunks;
    }
    return at;
}

int norm_and_clip(const sr_tensor *tensors, int n_tensors, float scale, float max_norm, bool clip, float *norm, void *workspace,
                  size_t workspace_bytes, hipStream_t stream) {
    if (n_tensors < 0 || (n_tensors > 0 && !tensors) || !norm || !workspace || (uintptr_t)workspace % 16 ||
        workspace_bytes < SR_GRAD_NORM_WORKSPACE || !std::isfinite(scale) || !std::isfinite(max_norm) || max_norm < 0.f)
        return SR_E_ARG;
    for (int i = 0; i < n_tensors; ++i) SR_TRY(check_tensor(tensors[i], clip));
    double *slots = (double *)workspace;
    TensorList l;
    int used = 0;
    for (int at = 0; at < n_tensors;) {
        at = take(tensors, n_tensors, at, &l);
        if (!l.tensors) continue;
        const int blocks = l.first[l.tensors] < kMostBlocks ? (int)l.first[l.tensors] : kMostBlocks;
        const bool fits = used + blocks <= kSlots;       // if not, at least kMostBlocks slots have been written
        square_sum_kernel<<<dim3(blocks), dim3(kNormThreads), 0, stream>>>(l, fits ? slots + used : slots, !fits);
        SR_HIP(hipGetLastError());
        if (fits) used += blocks;
    }
    norm_kernel<<<dim3(1), dim3(kNormThreads), 0, stream>>>(slots, used, scale, norm);
    SR_HIP(hipGetLastError());
    if (!clip) return SR_OK;
    for (int at = 0; at < n_tensors;) {
        at = take(tensors, n_tensors, at, &l);
        if (!l.tensors) continue;
        const int blocks = l.first[l.tensors] < kMostBlocks ? (int)l.first[l.tensors] : kMostBlocks;
        scale_kernel<<<dim3(blocks), dim3(kNormThreads), 0, stream>>>(l, slots, scale, max_norm);
        SR_HIP(hipGetLastError());
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
