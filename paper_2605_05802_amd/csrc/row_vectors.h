// 16 bytes at a time of float, bf16 or f16 data that may begin at any address its type allows, widened to single precision;
// and the sum over a workgroup.  Shared by the kernels of the update step.
#pragma once
#include <float.h>

#include "sr_internal.h"

namespace sr {

typedef _Float16 f16_t;

// The hardware reads and writes vectors at any address; the alignment says so to the compiler, which then splits nothing.
typedef uint32_t raw16 __attribute__((ext_vector_type(4), aligned(16)));
typedef uint32_t raw16_any __attribute__((ext_vector_type(4), aligned(2)));

template <typename T> struct Elem;
template <> struct Elem<float> {
    static constexpr int kPerVec = 4;
    static constexpr uint32_t kMinusInf = 0xff800000u;       // as many as fit 32 bits
    static __device__ __forceinline__ void widen(const raw16 &r, float *x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(r[i]);
    }
    static __device__ __forceinline__ raw16 narrow(const float *x) {
        raw16 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(x[i]);
        return r;
    }
};
template <> struct Elem<__bf16> {
    static constexpr int kPerVec = 8;
    static constexpr uint32_t kMinusInf = 0xff80ff80u;
    static __device__ __forceinline__ void widen(const raw16 &r, float *x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(r[i] << 16);
            x[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ raw16 narrow(const float *x) {
        raw16 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
        return r;
    }
};
template <> struct Elem<f16_t> {
    static constexpr int kPerVec = 8;
    static constexpr uint32_t kMinusInf = 0xfc00fc00u;
    typedef f16_t pair __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ void widen(const raw16 &r, float *x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const pair p = __builtin_bit_cast(pair, (uint32_t)r[i]);
            x[2 * i] = (float)p[0];
            x[2 * i + 1] = (float)p[1];
        }
    }
    static __device__ __forceinline__ raw16 narrow(const float *x) {
        raw16 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const pair p = {(f16_t)x[2 * i], (f16_t)x[2 * i + 1]};
            r[i] = __builtin_bit_cast(uint32_t, p);
        }
        return r;
    }
};

template <typename T> __device__ __forceinline__ raw16 load_vec(const T *p) { return *(const raw16_any *)p; }
// the same with the non-temporal hint, for data that the call does not touch again
template <typename T> __device__ __forceinline__ raw16 load_vec_once(const T *p) { return __builtin_nontemporal_load((const raw16_any *)p); }
template <typename T> __device__ __forceinline__ void store_vec_once(T *p, raw16 v) { __builtin_nontemporal_store(v, (raw16_any *)p); }

// 8 bytes
typedef uint32_t raw8 __attribute__((ext_vector_type(2), aligned(8)));
typedef uint32_t raw8_any __attribute__((ext_vector_type(2), aligned(2)));
template <typename T> __device__ __forceinline__ raw8 load_half_vec_once(const T *p) { return __builtin_nontemporal_load((const raw8_any *)p); }

// Reductions whose result every lane receives, by rotations within 16 lanes and swaps between them: no trip through LDS
template <typename F>
__device__ __forceinline__ float reduce_16(float x, F &&f) {
#define SR_ROTATE(n) f(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + n, 0xf, 0xf, false)))
    x = SR_ROTATE(8);
    x = SR_ROTATE(4);
    x = SR_ROTATE(2);
    return SR_ROTATE(1);
#undef SR_ROTATE
}
template <typename F>
__device__ __forceinline__ float reduce_64(float x, F &&f) {
    return row_reduce(reduce_16(x, f), f);
}

// A uniform address by a scalar load: it does not queue behind vector loads and stores.  Nothing that the kernel itself writes.
template <typename V> __device__ __forceinline__ V read_uniform(const V *p) {
    typedef std::conditional_t<sizeof(V) == 8, uint64_t, uint32_t> bits;
    return __builtin_bit_cast(V, *(const __attribute__((address_space(4))) bits *)p);
}

// Sum over the workgroup, in an order that depends on the thread number alone; valid in thread 0.  s: WAVES doubles of LDS,
// free to be overwritten.
template <int WAVES>
__device__ __forceinline__ double block_sum(double x, double *s) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off, 64);
    if (WAVES == 1) return x;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < WAVES; ++w) x += s[w];
    return x;
}

}  // namespace sr
