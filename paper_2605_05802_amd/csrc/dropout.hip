// Dropout with a mask that is never stored: out = [residual +] x m / (1 - p).  The backward pass is the same call on the gradient.
//
// Memory bounds it: x read, out written (and a residual read); the mask's two 64-bit products for four elements are hidden behind that.  One
// vector a thread, workgroups in the order of the memory: 8192 x 18944 bf16 113 us with the call, 5.5 TB/s, where a copy reaches 5.1; 203 rows
// of 1031 f16 3 us of 7 in the kernel.
#include "row_ops.h"

namespace sr {

int mask_args(const sr_mask *m, MaskArgs *a) {
    *a = MaskArgs{0, 0, 0, nullptr, 0, 1.f};
    if (!m) return SR_OK;
    if (!(m->p >= 0.f && m->p < 1.f) || (uintptr_t)m->step % 8) return SR_E_ARG;
    uint32_t drop = (uint32_t)((double)m->p * 65536.0 + 0.5);
    if (drop > 65535) drop = 65535;
    *a = MaskArgs{m->seed, m->mask, m->first_row, m->step, drop, (float)(65536.0 / (65536.0 - drop))};
    return SR_OK;
}

namespace {

struct DropArgs {
    const void *x, *residual;
    void *out;
    int64_t ld_x, ld_residual, ld_out;
    int rows, width, parts;          // workgroups of a row, 256 vectors each
    FastDiv by_parts;
    int lanes_shift;                 // log2 of the threads of a row where several rows share a workgroup
    MaskArgs mask;
};

template <typename T, typename R, bool ADD, int N>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs a) {
    int row, v;
    if (a.parts > 1) {
        row = quotient(blockIdx.x, a.by_parts);
        v = (int)(blockIdx.x - (unsigned)row * a.parts) * 256 + threadIdx.x;
    } else {
        row = (int)((blockIdx.x << (8 - a.lanes_shift)) + (threadIdx.x >> a.lanes_shift));
        v = threadIdx.x & ((1 << a.lanes_shift) - 1);
    }
    if (row >= a.rows) return;
    const Span s = span_of<N>(v, a.width);
    if (s.skip == N) return;
    Part<T, N> x;
    Part<R, N> r;
    x.load((const T *)a.x + row * a.ld_x + s.c);
    if (ADD) r.load((const R *)a.residual + row * a.ld_residual + s.c);
    float y[N];
    x.widen(y);
    if (a.mask.drop) drop_out<N>(mask_row(a.mask, mask_key(a.mask), row, a.width), s.c, a.width & 3, y);
    if (ADD) {
        float b[N];
        r.widen(b);
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] += b[j];
    }
    typedef std::conditional_t<ADD, R, T> O;
    store_span<N>((O *)a.out + row * a.ld_out, s, y);
}

template <typename T, typename R, bool ADD, int N>
int launch_dropout(DropArgs a, hipStream_t stream) {
    const int vecs = ceil_div(a.width, N);
    a.parts = ceil_div(vecs, 256);
    a.by_parts = fast_div(a.parts);
    a.lanes_shift = 0;
    while ((1 << a.lanes_shift) < vecs && a.lanes_shift < 8) ++a.lanes_shift;
    const int64_t blocks = a.parts > 1 ? (int64_t)a.rows * a.parts : ((int64_t)a.rows + (256 >> a.lanes_shift) - 1) >> (8 - a.lanes_shift);
    if (blocks > INT32_MAX / 256) return SR_E_LIMIT;
    dropout_kernel<T, R, ADD, N><<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(a);
    SR_HIP(hipGetLastError());
    return SR_OK;
}

}  // namespace
}  // namespace sr

extern "C" int sr_dropout(const sr_rows *x, const sr_rows *residual, const sr_rows *out, int rows, int width, const sr_mask *mask,
                          void *stream) {
    using namespace sr;
    const bool add = residual && residual->data;
    if (!x || !out || !mask || rows < 0 || width < 1) return SR_E_ARG;
    if (width > kMostDropWidth) return SR_E_LIMIT;
    DropArgs a{};
    SR_TRY(mask_args(mask, &a.mask));
    if (x->dtype < SR_F32 || x->dtype > SR_F16 || out->dtype != (add ? residual->dtype : x->dtype)) return SR_E_ARG;
    if (add && residual->dtype != x->dtype && residual->dtype != SR_F32) return SR_E_ARG;
    if (rows == 0) return SR_OK;
    if (!rows_fit(*x, width, SR_F16) || !rows_fit(*out, width, SR_F16) || (add && !rows_fit(*residual, width, SR_F16))) return SR_E_ARG;
    if (!in_place_or_apart(*out, *x) || (add && !in_place_or_apart(*out, *residual))) return SR_E_ARG;
    a.x = x->data;
    a.ld_x = x->ld;
    a.residual = add ? residual->data : nullptr;
    a.ld_residual = add ? residual->ld : 0;
    a.out = out->data;
    a.ld_out = out->ld;
    a.rows = rows;
    a.width = width;
    return with_row_types(x->dtype, out->dtype, [&](auto *t, auto *r) -> int {
        typedef std::remove_pointer_t<decltype(t)> T;
        typedef std::remove_pointer_t<decltype(r)> R;
        constexpr int N = sizeof(R) == 4 ? 4 : 8;
        const bool narrow = width < 8;
        if (add) return narrow ? launch_dropout<T, R, true, 1>(a, (hipStream_t)stream) : launch_dropout<T, R, true, N>(a, (hipStream_t)stream);
        if constexpr (std::is_same_v<T, R>)
            return narrow ? launch_dropout<T, T, false, 1>(a, (hipStream_t)stream) : launch_dropout<T, T, false, N>(a, (hipStream_t)stream);
        return SR_E_ARG;
    });
}
