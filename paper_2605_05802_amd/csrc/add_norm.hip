// Residual + branch and the root-mean-square norm of the sum, for training: the sum and 1 / sqrt(mean + eps) stay for the backward pass.
//
// h = residual + dropout(x), rounded to the residual's type; out = h * rstd * gain, rstd = 1 / sqrt(mean(h^2) + eps), of h as it is stored,
// so that the backward pass, which reads it, differentiates what was computed.  Memory bounds it: x and residual read, h and out
// written.  A row lies in the registers of its workgroup (of a wavefront, up to 64
// vectors, of 16 or 32 lanes, up to 16 or 32) between the sum and its use.
//
// 8192 rows of 3584 bf16 beside fp32, into e4m3 with a scale for 128 columns: 62 us with the call, 5.2 TB/s; 128 rows 4 us in the kernel, 1531
// rows of 2047 f16 with dropout 8.8, 7.7 without: one round of workgroups that load, reduce and store.  One, two or four vectors a thread are even at
// these sizes.
//
// Output in 8 bits: a scale for a row or for 32, 64 or 128 of its columns, max |out| / (largest finite value), which the block's columns
// are divided by; adjacent lanes hold a block and find its largest value between them.
#include <cmath>

#include "row_ops.h"

namespace sr {
namespace {

struct NormRowArgs {
    const void *x, *residual, *gain;
    void *total, *out;
    int64_t ld_x, ld_residual, ld_total, ld_out;
    float *rstd, *scales;
    int rows, width;
    int has_x, gain_single;          // x: read in any case, the gain where there is none
    int e5m2, block_lanes, blocks;   // lanes of a block, 0: the row; blocks of a row
    float eps;
    MaskArgs mask;
};

// Largest value over aligned groups of `lanes` adjacent lanes: 4 to 32
__device__ __forceinline__ float max_of_lanes(float x, int lanes) {
#define SR_MAX_DPP(ctrl) x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl, 0xf, 0xf, false)))
    SR_MAX_DPP(0xB1);                // lanes 1 0 3 2
    SR_MAX_DPP(0x4E);                // lanes 2 3 0 1
    if (lanes >= 8) SR_MAX_DPP(0x141);                   // of eight, backwards
    if (lanes >= 16) SR_MAX_DPP(0x140);                  // of sixteen, backwards
#undef SR_MAX_DPP
    if (lanes >= 32) {
        const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
    }
    return x;
}

// Two of them in the low half; the instruction rounds to nearest even, and what a scale was made for is within range
__device__ __forceinline__ uint32_t pack_8bit(float a, float b, bool e5m2) {
    return (uint32_t)(e5m2 ? __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false) : __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false)) & 0xffffu;
}

template <int N>
__device__ __forceinline__ void store_bytes(uint8_t *row, const Span &s, const float *y, bool e5m2) {
    uint32_t w[(N + 3) / 4];
    if constexpr (N == 1) w[0] = pack_8bit(y[0], 0.f, e5m2);
    else
#pragma unroll
        for (int i = 0; i < N / 4; ++i) w[i] = pack_8bit(y[4 * i], y[4 * i + 1], e5m2) | pack_8bit(y[4 * i + 2], y[4 * i + 3], e5m2) << 16;
    if (s.skip == 0) {
        if constexpr (N == 1) row[s.c] = (uint8_t)w[0];
        else if constexpr (N == 4) *(raw4_any *)(row + s.c) = w[0];
        else *(raw8_bytes *)(row + s.c) = raw8_bytes{w[0], w[1]};
    } else {
#pragma unroll
        for (int j = 1; j < N; ++j)
            if (j >= s.skip) row[s.c + j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
    }
}

// LANES: of a row that is a part of a wavefront or a whole one; 0: a workgroup
template <typename T, typename R, bool BYTES, int N, int NV, int LANES>
__global__ __launch_bounds__(LANES ? 256 : 1024) void add_norm_kernel(NormRowArgs a) {
    __shared__ float s_sum[16], s_max[16];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    const int row = LANES && LANES < 64 ? (int)(blockIdx.x * (256 / LANES) + threadIdx.x / LANES)
                                        : __builtin_amdgcn_readfirstlane(LANES ? (int)blockIdx.x * 4 + wave : (int)blockIdx.x);
    if (LANES && row >= a.rows) return;
    const int first = LANES ? (int)threadIdx.x & (LANES - 1) : (int)threadIdx.x, step = (int)blockDim.x;
    const T *x = (const T *)a.x + row * a.ld_x;
    const R *residual = (const R *)a.residual + row * a.ld_residual;

    Span at[NV];
    Part<T, N> xp[NV];
    Part<R, N> rp[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        at[i] = span_of<N>(first + i * step, a.width);
        rp[i].load(residual + at[i].c);
        xp[i].load(x + at[i].c);
    }
    float g[NV][N];
    if (a.gain_single) {
        Part<float, N> p[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) p[i].load((const float *)a.gain + at[i].c);
#pragma unroll
        for (int i = 0; i < NV; ++i) p[i].widen(g[i]);
    } else {
        Part<T, N> p[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) p[i].load((const T *)a.gain + at[i].c);
#pragma unroll
        for (int i = 0; i < NV; ++i) p[i].widen(g[i]);
    }

    float h[NV][N], sum = 0.f;
    const uint64_t key = mask_key(a.mask);
    const MaskRow mask = mask_row(a.mask, key, row, a.width);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float b[N];
        xp[i].widen(b);
        rp[i].widen(h[i]);
        if (a.mask.drop) drop_out<N>(mask, at[i].c, a.width & 3, b);
#pragma unroll
        for (int j = 0; j < N; ++j) h[i][j] += a.has_x ? b[j] : 0.f;
        if (sizeof(R) == 2) {
            rp[i].narrow(h[i]);
            rp[i].widen(h[i]);
        }
        if (a.total) store_span<N>((R *)a.total + row * a.ld_total, at[i], h[i]);
#pragma unroll
        for (int j = 0; j < N; ++j) sum = j >= at[i].skip ? fmaf(h[i][j], h[i][j], sum) : sum;
    }
    sum = reduce_lanes<LANES>(sum, [](float p, float q) { return p + q; });
    if (!LANES) {
        if (lane == 0) s_sum[wave] = sum;
        __syncthreads();
        sum = s_sum[0];
        for (int w = 1; w < waves; ++w) sum += s_sum[w];
    }
    const float rstd = 1.0f / sqrtf(sum / (float)a.width + a.eps);
    if (a.rstd && first == 0) a.rstd[row] = rstd;

    float y[NV][N];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) y[i][j] = h[i][j] * rstd * g[i][j];
    if constexpr (!BYTES) {
#pragma unroll
        for (int i = 0; i < NV; ++i) store_span<N>((T *)a.out + row * a.ld_out, at[i], y[i]);
    } else {
        const float largest = a.e5m2 ? 57344.f : 448.f;
        float most[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            most[i] = 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j) most[i] = j >= at[i].skip ? fmaxf(most[i], fabsf(y[i][j])) : most[i];
        }
        if (a.block_lanes) {
#pragma unroll
            for (int i = 0; i < NV; ++i) most[i] = max_of_lanes(most[i], a.block_lanes);
        } else {
#pragma unroll
            for (int i = 1; i < NV; ++i) most[0] = fmaxf(most[0], most[i]);
            most[0] = reduce_lanes<LANES>(most[0], [](float p, float q) { return fmaxf(p, q); });
            if (!LANES) {
                if (lane == 0) s_max[wave] = most[0];
                __syncthreads();
                for (int w = 0; w < waves; ++w) most[0] = fmaxf(most[0], s_max[w]);
            }
#pragma unroll
            for (int i = 1; i < NV; ++i) most[i] = most[0];
        }
        float *scales = a.scales + (size_t)row * a.blocks;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = first + i * step;
            // not below the smallest normal number: a block of zeros has zeros as codes
            const float scale = fmaxf(most[i] / largest, FLT_MIN);
#pragma unroll
            for (int j = 0; j < N; ++j) y[i][j] /= scale;
            store_bytes<N>((uint8_t *)a.out + row * a.ld_out, at[i], y[i], a.e5m2);
            if (at[i].skip < N && (a.block_lanes ? (v & (a.block_lanes - 1)) == 0 : v == 0))
                scales[a.block_lanes ? v / a.block_lanes : 0] = scale;
        }
    }
}

template <typename T, typename R, bool BYTES, int N>
int launch_add_norm(const NormRowArgs &a, const RowShape &s, hipStream_t stream) {
    const int each = s.lanes ? 256 / s.lanes : 1;
    const dim3 grid((unsigned)(((int64_t)a.rows + each - 1) / each));
    if (s.lanes == 16) add_norm_kernel<T, R, BYTES, N, 1, 16><<<grid, dim3(256), 0, stream>>>(a);
    else if constexpr (N > 1) {
        if (s.lanes == 32) add_norm_kernel<T, R, BYTES, N, 1, 32><<<grid, dim3(256), 0, stream>>>(a);
        else if (s.lanes) add_norm_kernel<T, R, BYTES, N, 1, 64><<<grid, dim3(256), 0, stream>>>(a);
        else if (s.vecs == 1) add_norm_kernel<T, R, BYTES, N, 1, 0><<<grid, dim3(s.threads), 0, stream>>>(a);
        else if (s.vecs == 2) add_norm_kernel<T, R, BYTES, N, 2, 0><<<grid, dim3(s.threads), 0, stream>>>(a);
        else if constexpr (N == 4) add_norm_kernel<T, R, BYTES, N, 4, 0><<<grid, dim3(s.threads), 0, stream>>>(a);
    }
    SR_HIP(hipGetLastError());
    return SR_OK;
}

static_assert(sizeof(sr_rows) == 24 && sizeof(sr_norm_rows) == 152, "the binding packs them by hand");
int add_norm(const sr_norm_rows *x, hipStream_t stream) {
    if (!x || x->rows < 0 || x->width < 1 || !std::isfinite(x->eps) || x->eps < 0.f) return SR_E_ARG;
    const int dtype = x->x.dtype, residual = x->residual.dtype;
    const bool bytes = x->out.dtype == SR_E4M3 || x->out.dtype == SR_E5M2;
    NormRowArgs a{};
    SR_TRY(mask_args(x->dropout, &a.mask));
    if (dtype < SR_F32 || dtype > SR_F16 || (residual != dtype && residual != SR_F32)) return SR_E_ARG;
    if ((!bytes && x->out.dtype != dtype) || (x->gain_dtype != dtype && x->gain_dtype != SR_F32)) return SR_E_ARG;
    const int block = x->scale_block;
    if (bytes ? block != 0 && block != 32 && block != 64 && block != 128 : block != 0) return SR_E_ARG;
    if (x->total.data && x->total.dtype != residual) return SR_E_ARG;
    if (x->width > kMostNormWidth) return SR_E_LIMIT;
    if (x->rows == 0) return SR_OK;
    if (!rows_fit(x->residual, x->width, SR_F16) || !rows_fit(x->out, x->width, SR_E5M2)) return SR_E_ARG;
    if ((x->x.data && !rows_fit(x->x, x->width, SR_F16)) || (x->total.data && !rows_fit(x->total, x->width, SR_F16))) return SR_E_ARG;
    if (!x->gain || (uintptr_t)x->gain % elem_bytes(x->gain_dtype) || (uintptr_t)x->rstd % 4 || (uintptr_t)x->scales % 4) return SR_E_ARG;
    if (bytes != (x->scales != nullptr)) return SR_E_ARG;
    if (!in_place_or_apart(x->total, x->residual) || !in_place_or_apart(x->out, x->x) || x->total.data == x->out.data ||
        x->out.data == x->residual.data || (x->total.data && x->total.data == x->x.data))
        return SR_E_ARG;
    const bool single = dtype == SR_F32 || residual == SR_F32;
    const RowShape shape = norm_shape(x->width, single);
    if ((int64_t)x->rows * shape.threads > UINT32_MAX - 255) return SR_E_LIMIT;
    a.has_x = x->x.data != nullptr;
    const BranchRows branch = branch_rows(x->x.data, x->x.ld, x->gain);
    a.x = branch.data;
    a.ld_x = branch.ld;
    if (!a.has_x) a.mask.drop = 0;
    a.residual = x->residual.data;
    a.ld_residual = x->residual.ld;
    a.gain = x->gain;
    a.gain_single = x->gain_dtype == SR_F32;
    a.total = x->total.data;
    a.ld_total = x->total.ld;
    a.out = x->out.data;
    a.ld_out = x->out.ld;
    a.rstd = x->rstd;
    a.scales = x->scales;
    a.rows = x->rows;
    a.width = x->width;
    a.e5m2 = x->out.dtype == SR_E5M2;
    // a block that holds the row is the row
    a.block_lanes = block && block < x->width ? block / shape.per_vec : 0;
    a.blocks = block ? ceil_div(x->width, block) : 1;
    a.eps = x->eps;
    return with_row_types(dtype, residual, [&](auto *t, auto *r) -> int {
        typedef std::remove_pointer_t<decltype(t)> T;
        typedef std::remove_pointer_t<decltype(r)> R;
        constexpr int N = sizeof(R) == 4 ? 4 : 8;
        if (shape.per_vec == 1)
            return bytes ? launch_add_norm<T, R, true, 1>(a, shape, stream) : launch_add_norm<T, R, false, 1>(a, shape, stream);
        return bytes ? launch_add_norm<T, R, true, N>(a, shape, stream) : launch_add_norm<T, R, false, N>(a, shape, stream);
    });
}

}  // namespace
}  // namespace sr

extern "C" int sr_add_norm(const sr_norm_rows *rows, void *stream) { return sr::add_norm(rows, (hipStream_t)stream); }
