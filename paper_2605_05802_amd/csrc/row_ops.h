// Parts of rows in registers, and the masks of dropout: shared by the row operators of training.
#pragma once
#include "row_plan.h"
#include "row_vectors.h"
#include "splitmix.h"

namespace sr {

typedef uint32_t raw4_any __attribute__((aligned(1)));
typedef uint32_t raw8_bytes __attribute__((ext_vector_type(2), aligned(1)));

// N elements of a row, 1, 4 or 8, as they lie in memory, at any address that their type allows
template <typename T, int N>
struct Part {
    static constexpr int kBytes = N * (int)sizeof(T), kQuads = kBytes / 16;
    static_assert(N == 1 || kBytes == 8 || kBytes % 16 == 0, "width");
    union {
        raw16 q[kQuads ? kQuads : 1];
        raw8 h;
        T one;
    };
    __device__ __forceinline__ Part() {}
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (N == 1) one = *p;
        else if constexpr (kBytes == 8) h = *(const raw8_any *)p;
        else
#pragma unroll
            for (int i = 0; i < kQuads; ++i) q[i] = *((const raw16_any *)p + i);
    }
    __device__ __forceinline__ void store(T *p) const {
        if constexpr (N == 1) *p = one;
        else if constexpr (kBytes == 8) *(raw8_any *)p = h;
        else
#pragma unroll
            for (int i = 0; i < kQuads; ++i) *((raw16_any *)p + i) = q[i];
    }
    __device__ __forceinline__ void widen(float *x) const {
        if constexpr (N == 1) x[0] = (float)one;
        else if constexpr (kBytes == 8) {
            const raw16 r = {h[0], h[1], 0u, 0u};
            float y[8];
            Elem<T>::widen(r, y);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = y[i];
        } else {
#pragma unroll
            for (int i = 0; i < kQuads; ++i) Elem<T>::widen(q[i], x + i * Elem<T>::kPerVec);
        }
    }
    __device__ __forceinline__ void narrow(const float *x) {
        if constexpr (N == 1) one = (T)x[0];
        else if constexpr (kBytes == 8) {
            const float y[8] = {x[0], x[1], x[2], x[3], 0.f, 0.f, 0.f, 0.f};
            const raw16 r = Elem<T>::narrow(y);
            h[0] = r[0];
            h[1] = r[1];
        } else {
#pragma unroll
            for (int i = 0; i < kQuads; ++i) q[i] = Elem<T>::narrow(x + i * Elem<T>::kPerVec);
        }
    }
};

// Vector v of a row of `width` >= N columns: columns c .. c + N - 1, of which the first `skip` belong to the vector before (the row's last
// vector lies over it where the width is no multiple of N) and `skip` = N behind the row's end.
struct Span {
    int c, skip;
};
template <int N>
__device__ __forceinline__ Span span_of(int v, int width) {
    const int at = v * N, c = min(at, width - N), over = at - c;
    return Span{c, min(over, N)};
}
template <int N, typename T>
__device__ __forceinline__ void store_span(T *row, const Span &s, const float *x) {
    if (s.skip == 0) {
        Part<T, N> p;
        p.narrow(x);
        p.store(row + s.c);
    } else {
#pragma unroll
        for (int j = 1; j < N; ++j)                  // the whole vector where skip is 0
            if (j >= s.skip) row[s.c + j] = (T)x[j];
    }
}

// What lanes of this wavefront wrote to LDS before is there for its other lanes behind it.  The hardware keeps a wavefront's LDS accesses in
// order and needs nothing for that; the compiler, which sees one lane, has to be told.  All lanes come here.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Over the lanes of a row: 16 or 32 of them or the wavefront
template <int LANES, typename F>
__device__ __forceinline__ float reduce_lanes(float x, F &&f) {
    if (LANES != 16 && LANES != 32) return reduce_64(x, f);
    x = reduce_16(x, f);
    if (LANES == 16) return x;
    const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return f(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

// ---------------------------------------------------------------------------------------------
// dropout
// ---------------------------------------------------------------------------------------------
// Element (row, column) of a mask has the 16 bits (column % 4) of word (row * ceil(width / 4) + column / 4) of a SplitMix64 stream, and
// goes if they are below `drop` = min(65535, round(65536 p)).  16 bits make four elements of a word, whose two 64-bit products are what a mask costs;
// the kept ones are multiplied by 65536 / (65536 - drop), the reciprocal of the share that these bits keep.
struct MaskArgs {
    uint64_t seed, which, first_row;
    const uint64_t *step;        // added to `which`, or null
    uint32_t drop;               // 0: nothing is dropped
    float keep;
};
// host side: SR_E_ARG for a senseless one; null is no dropout
int mask_args(const sr_mask *m, MaskArgs *a);

struct MaskRow {
    uint64_t at;                 // key + counter of the row's first word
    uint32_t drop;
    float keep;
};
__device__ __forceinline__ uint64_t mask_key(const MaskArgs &m) {
    return m.drop ? smx_key(m.seed, m.which + (m.step ? read_uniform(m.step) : 0)) : 0;
}
__device__ __forceinline__ MaskRow mask_row(const MaskArgs &m, uint64_t key, uint64_t row, int width) {
    return MaskRow{key + ((m.first_row + row) * (uint64_t)((width + 3) >> 2) + 1ULL) * kGolden, m.drop, m.keep};
}
// x[j] of columns c + j, N of them.  A column c that is no multiple of four has bits of one more word: in rows whose width is none.
template <int N>
__device__ __forceinline__ void drop_out(const MaskRow &m, int c, bool ragged, float *x) {
    constexpr int kWords = (N + 3) / 4;
    uint64_t w[kWords];
    const uint64_t at = m.at + (uint64_t)(c >> 2) * kGolden;
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = smx_finalize(at + (uint64_t)i * kGolden);
    if (N == 1) {
        w[0] >>= 16 * (c & 3);
    } else if (ragged) {
        const int shift = 16 * (c & 3);
        if (shift) {                                 // a row's last vector alone: no lane of most wavefronts
            const uint64_t more = smx_finalize(at + (uint64_t)kWords * kGolden);
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = w[i] >> shift | (i + 1 < kWords ? w[i + 1] : more) << (64 - shift);
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const uint32_t u = (uint32_t)(w[j >> 2] >> (16 * (j & 3))) & 0xffffu;
        x[j] = u < m.drop ? 0.f : x[j] * m.keep;
    }
}

// f(T{}, R{}) for the types of a branch and of the residual beside it, which is of the same type or in single precision
template <typename F>
int with_row_types(int dtype, int residual, F &&f) {
    if (residual != dtype && residual != SR_F32) return SR_E_ARG;
    if (dtype == SR_F32) return f((float *)nullptr, (float *)nullptr);
    if (dtype == SR_BF16) return residual == SR_F32 ? f((__bf16 *)nullptr, (float *)nullptr) : f((__bf16 *)nullptr, (__bf16 *)nullptr);
    if (dtype == SR_F16) return residual == SR_F32 ? f((f16_t *)nullptr, (float *)nullptr) : f((f16_t *)nullptr, (f16_t *)nullptr);
    return SR_E_ARG;
}

inline int elem_bytes(int dtype) { return dtype == SR_F32 ? 4 : dtype == SR_BF16 || dtype == SR_F16 ? 2 : 1; }
// Rows that a call may read or write: there, of a type from SR_F32 to `last`, rows that do not run into each other
inline bool rows_fit(const sr_rows &r, int width, int last) {
    return r.data && r.dtype >= SR_F32 && r.dtype <= last && (uintptr_t)r.data % elem_bytes(r.dtype) == 0 && r.ld >= width &&
           r.ld <= ((int64_t)1 << 40);
}
// An output that begins where an input does is the input, element by element
inline bool in_place_or_apart(const sr_rows &out, const sr_rows &in) {
    return !out.data || out.data != in.data || (out.ld == in.ld && out.dtype == in.dtype);
}

}  // namespace sr
