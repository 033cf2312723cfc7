// Gradients of residual + branch and the root-mean-square norm of their sum.
//
// With dy the gradient of the output, h the stored sum, n = h * rstd: g = dy * gain, dh = rstd * (g - n * mean(g n)) + d_total, where
// d_total arrives at the sum from behind it; d_residual = dh, d_x = dropout(dh), d_gain = sum over rows of dy * n.
//
// Memory bounds it: dy, h and d_total read, d_residual and d_x written.  Workgroups (wavefronts, for rows of up to 64 vectors, two and four at a time up to 32 and 16) take
// rows in turn, hold the next row's vectors while they reduce and write the one before, and keep their share of d_gain in registers;
// a second kernel adds the shares up in the order of their numbers, so that the sum is the same bit for bit from call to call.  Of few rows
// the gain's gradient is added up from the rows themselves, by other workgroups of the same launch.
// 16384 rows of 3584 bf16 beside fp32, with dropout: 183 + 5 us, 5.1 TB/s of 588 MB read and 360 written.
#include "row_ops.h"

namespace sr {
namespace {

struct NormGradArgs {
    const void *d_out, *total, *d_total, *gain;
    void *d_residual, *d_x, *d_gain;
    int64_t ld_d_out, ld_total, ld_d_total, ld_d_residual, ld_d_x;
    const float *rstd;
    float *parts;                    // [n_parts][width]
    int rows, width, n_parts;
    int has_d_total, gain_single, gain_grad_single, gain_grad_half, accumulate;
    MaskArgs mask;
};

// A gain's gradient, sixteen columns a workgroup: x(p, c) added up over p < n, by groups of lanes that take the numbers in turn, then over the
// groups of a wavefront and over the wavefronts.  s: 16 x kGainColumns floats of LDS.
constexpr int kGainColumns = 16;
template <typename F>
__device__ __forceinline__ void gain_columns(const NormGradArgs &a, int block, int n, float (*s)[kGainColumns], F &&x) {
    const int groups = (int)blockDim.x / kGainColumns, group = (int)threadIdx.x / kGainColumns, i = (int)threadIdx.x % kGainColumns;
    const int c = block * kGainColumns + i, at = min(c, a.width - 1);
    float sum = 0.f;
    for (int p = group; p < n; p += 8 * groups) {
        float y[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) y[u] = x(min(p + u * groups, n - 1), at);
#pragma unroll
        for (int u = 0; u < 8; ++u) sum += p + u * groups < n ? y[u] : 0.f;
    }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if ((threadIdx.x & 63) < kGainColumns) s[threadIdx.x >> 6][i] = sum;
    __syncthreads();
    if (group != 0 || c >= a.width) return;
    sum = s[0][i];
    for (int w = 1; w < (int)blockDim.x >> 6; ++w) sum += s[w][i];
    if (a.gain_grad_single) {
        float *to = (float *)a.d_gain + c;
        *to = a.accumulate ? *to + sum : sum;
    } else if (a.gain_grad_half) {
        f16_t *to = (f16_t *)a.d_gain + c;
        *to = (f16_t)(a.accumulate ? (float)*to + sum : sum);
    } else {
        __bf16 *to = (__bf16 *)a.d_gain + c;
        *to = (__bf16)(a.accumulate ? (float)*to + sum : sum);
    }
}

// From the shares of add_norm_grad_kernel's workgroups
__global__ __launch_bounds__(1024) void gain_grad_kernel(NormGradArgs a) {
    __shared__ float s[16][kGainColumns];
    gain_columns(a, (int)blockIdx.x, a.n_parts, s, [&](int p, int c) { return a.parts[(size_t)p * a.width + c]; });
}

template <typename T, typename R, int N, int NV>
struct GradRow {
    Part<T, N> dy[NV];
    Part<R, N> h[NV], dt[NV];
    float rstd;

    __device__ __forceinline__ void load(const NormGradArgs &a, int row, const Span *at) {
        const T *d_out = (const T *)a.d_out + row * a.ld_d_out;
        const R *total = (const R *)a.total + row * a.ld_total, *d_total = (const R *)a.d_total + row * a.ld_d_total;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            dy[i].load(d_out + at[i].c);
            h[i].load(total + at[i].c);
            dt[i].load(d_total + at[i].c);
        }
        rstd = a.rstd[row];
    }
};

// LANES: of a row that is a part of a wavefront or a whole one; 0: a workgroup
template <typename T, typename R, int N, int NV, int LANES>
__global__ __launch_bounds__(LANES ? 256 : 1024) void add_norm_grad_kernel(NormGradArgs a) {
    __shared__ float s_sum[2][16];
    const int row_blocks = LANES ? (a.n_parts + 3) / 4 : a.n_parts;
    if ((int)blockIdx.x >= row_blocks) {             // few rows: the gain's gradient from the rows themselves
        __shared__ float s[16][kGainColumns];
        gain_columns(a, (int)blockIdx.x - row_blocks, a.rows, s, [&](int r, int c) {
            return (float)((const T *)a.d_out)[r * a.ld_d_out + c] * ((float)((const R *)a.total)[r * a.ld_total + c] * a.rstd[r]);
        });
        return;
    }
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    const int part = __builtin_amdgcn_readfirstlane(LANES ? (int)blockIdx.x * 4 + wave : (int)blockIdx.x);
    if (LANES && part >= a.n_parts) return;
    const int first = LANES ? lane & (LANES - 1) : (int)threadIdx.x, step = (int)blockDim.x;
    constexpr int kBeside = LANES ? 64 / LANES : 1;              // rows beside each other
    const int begin = part * kBeside + (LANES ? lane / LANES : 0), stride = a.n_parts * kBeside;
    Span at[NV];
    float gain[NV][N], d_gain[NV][N];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        at[i] = span_of<N>(first + i * step, a.width);
        if (a.gain_single) {
            Part<float, N> p;
            p.load((const float *)a.gain + at[i].c);
            p.widen(gain[i]);
        } else {
            Part<T, N> p;
            p.load((const T *)a.gain + at[i].c);
            p.widen(gain[i]);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) d_gain[i][j] = 0.f;
    }
    const uint64_t key = mask_key(a.mask);

    // the next row's vectors beside this one's, where registers hold both
    constexpr bool kAhead = N * NV <= 8;
    GradRow<T, R, N, NV> next;
    if (kAhead) next.load(a, min(begin, a.rows - 1), at);
    int turn = 0;
    for (int row = begin; row < a.rows; row += stride, turn ^= 1) {
        if (!kAhead) next.load(a, row, at);
        const GradRow<T, R, N, NV> x = next;
        if (kAhead) next.load(a, min(row + stride, a.rows - 1), at);
        float g[NV][N], n[NV][N], sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float dy[N];
            x.dy[i].widen(dy);
            x.h[i].widen(n[i]);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                n[i][j] *= x.rstd;
                g[i][j] = dy[j] * gain[i][j];
                d_gain[i][j] = fmaf(dy[j], n[i][j], d_gain[i][j]);
                sum += j >= at[i].skip ? g[i][j] * n[i][j] : 0.f;
            }
        }
        sum = reduce_lanes<LANES>(sum, [](float p, float q) { return p + q; });
        if (!LANES) {
            if (lane == 0) s_sum[turn][wave] = sum;
            __syncthreads();
            sum = s_sum[turn][0];
            for (int w = 1; w < waves; ++w) sum += s_sum[turn][w];
        }
        const float mean = sum / (float)a.width;
        const MaskRow mask = mask_row(a.mask, key, row, a.width);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float dt[N];
            x.dt[i].widen(dt);
#pragma unroll
            for (int j = 0; j < N; ++j) g[i][j] = x.rstd * (g[i][j] - n[i][j] * mean) + (a.has_d_total ? dt[j] : 0.f);
            if (a.d_residual) store_span<N>((R *)a.d_residual + row * a.ld_d_residual, at[i], g[i]);
            if (a.d_x) {
                if (a.mask.drop) drop_out<N>(mask, at[i].c, a.width & 3, g[i]);
                store_span<N>((T *)a.d_x + row * a.ld_d_x, at[i], g[i]);
            }
        }
    }
    if (!a.parts) return;
    if (kBeside > 1) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (kBeside == 4) d_gain[0][j] += __shfl_xor(d_gain[0][j], 16, 64);
            d_gain[0][j] += __shfl_xor(d_gain[0][j], 32, 64);
        }
        if (lane >= LANES) return;
    }
    float *to = a.parts + (size_t)part * a.width;
#pragma unroll
    for (int i = 0; i < NV; ++i) store_span<N>(to, at[i], d_gain[i]);
}

template <typename T, typename R, int N>
int launch_add_norm_grad(const NormGradArgs &a, const RowShape &s, hipStream_t stream) {
    const int more = a.d_gain && !a.parts ? ceil_div(a.width, kGainColumns) : 0;
    const dim3 grid((s.lanes ? ceil_div(a.n_parts, 4) : a.n_parts) + more);
    if (s.lanes == 16) add_norm_grad_kernel<T, R, N, 1, 16><<<grid, dim3(256), 0, stream>>>(a);
    else if constexpr (N > 1) {
        if (s.lanes == 32) add_norm_grad_kernel<T, R, N, 1, 32><<<grid, dim3(256), 0, stream>>>(a);
        else if (s.lanes) add_norm_grad_kernel<T, R, N, 1, 64><<<grid, dim3(256), 0, stream>>>(a);
        else if (s.vecs == 1) add_norm_grad_kernel<T, R, N, 1, 0><<<grid, dim3(s.threads), 0, stream>>>(a);
        else if (s.vecs == 2) add_norm_grad_kernel<T, R, N, 2, 0><<<grid, dim3(s.threads), 0, stream>>>(a);
        else if constexpr (N == 4) add_norm_grad_kernel<T, R, N, 4, 0><<<grid, dim3(s.threads), 0, stream>>>(a);
    }
    SR_HIP(hipGetLastError());
    return SR_OK;
}

static_assert(sizeof(sr_norm_grad_rows) == 176, "the binding packs it by hand");
int add_norm_grad(const sr_norm_grad_rows *x, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!x || x->rows < 0 || x->width < 1) return SR_E_ARG;
    const int dtype = x->d_out.dtype, residual = x->total.dtype;
    NormGradArgs a{};
    SR_TRY(mask_args(x->dropout, &a.mask));
    if (dtype < SR_F32 || dtype > SR_F16 || (residual != dtype && residual != SR_F32)) return SR_E_ARG;
    if (x->gain_dtype != dtype && x->gain_dtype != SR_F32) return SR_E_ARG;
    if (x->d_gain && x->d_gain_dtype != dtype && x->d_gain_dtype != SR_F32) return SR_E_ARG;
    if (x->rows > 0 && !x->d_residual.data && !x->d_x.data && !x->d_gain) return SR_E_ARG;
    if (x->width > kMostNormWidth) return SR_E_LIMIT;
    if (x->d_gain && ((uintptr_t)x->d_gain % elem_bytes(x->d_gain_dtype) || x->d_gain == x->gain)) return SR_E_ARG;
    if (x->rows > 0) {
        if (!rows_fit(x->d_out, x->width, SR_F16) || !rows_fit(x->total, x->width, SR_F16)) return SR_E_ARG;
        for (const sr_rows *r : {&x->d_total, &x->d_residual})
            if (r->data && (r->dtype != residual || !rows_fit(*r, x->width, SR_F16))) return SR_E_ARG;
        if (x->d_x.data && (x->d_x.dtype != dtype || !rows_fit(x->d_x, x->width, SR_F16))) return SR_E_ARG;
        if (!x->rstd || (uintptr_t)x->rstd % 4 || !x->gain || (uintptr_t)x->gain % elem_bytes(x->gain_dtype)) return SR_E_ARG;
        // in the place of what arrives from behind, and of nothing else
        if (!in_place_or_apart(x->d_residual, x->d_total) || !in_place_or_apart(x->d_x, x->d_out)) return SR_E_ARG;
        for (const void *out : {x->d_residual.data, x->d_x.data})
            if (out && (out == x->total.data || out == x->gain || out == x->d_gain)) return SR_E_ARG;
        if ((x->d_residual.data && (x->d_residual.data == x->d_x.data || x->d_residual.data == x->d_out.data)) ||
            (x->d_x.data && x->d_x.data == x->d_total.data))
            return SR_E_ARG;
    }
    const bool single = dtype == SR_F32 || residual == SR_F32;
    const RowShape shape = norm_shape(x->width, single);
    if ((int64_t)x->rows * shape.threads > UINT32_MAX - 255) return SR_E_LIMIT;      // as forward; row numbers then have room above them
    a.n_parts = norm_grad_parts(x->rows, shape);
    if (x->d_gain && (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < SR_NORM_GRAD_WORKSPACE(x->rows, x->width))) return SR_E_ARG;
    a.d_out = x->d_out.data;
    a.ld_d_out = x->d_out.ld;
    a.total = x->total.data;
    a.ld_total = x->total.ld;
    a.has_d_total = x->d_total.data != nullptr;
    a.d_total = a.has_d_total ? x->d_total.data : x->total.data;
    a.ld_d_total = a.has_d_total ? x->d_total.ld : x->total.ld;
    a.d_residual = x->d_residual.data;
    a.ld_d_residual = x->d_residual.ld;
    a.d_x = x->d_x.data;
    a.ld_d_x = x->d_x.ld;
    a.gain = x->gain;
    a.gain_single = x->gain_dtype == SR_F32;
    a.d_gain = x->d_gain;
    a.gain_grad_single = x->d_gain_dtype == SR_F32;
    a.accumulate = x->accumulate != 0;
    a.rstd = x->rstd;
    a.gain_grad_half = x->d_gain_dtype == SR_F16;
    // the workgroups for the gain read d_out while others write d_x
    const bool direct = x->rows > 0 && gain_grad_direct(x->rows, x->width) && x->d_x.data != x->d_out.data;
    a.parts = x->d_gain && !direct ? (float *)workspace : nullptr;
    a.rows = x->rows;
    a.width = x->width;
    return with_row_types(dtype, residual, [&](auto *t, auto *r) -> int {
        typedef std::remove_pointer_t<decltype(t)> T;
        typedef std::remove_pointer_t<decltype(r)> R;
        constexpr int N = sizeof(R) == 4 ? 4 : 8;
        if (a.rows > 0)
            SR_TRY((shape.per_vec == 1 ? launch_add_norm_grad<T, R, 1>(a, shape, stream) : launch_add_norm_grad<T, R, N>(a, shape, stream)));
        if (!a.parts) return SR_OK;
        gain_grad_kernel<<<dim3(ceil_div(a.width, kGainColumns)), dim3(1024), 0, stream>>>(a);
        SR_HIP(hipGetLastError());
        return SR_OK;
    });
}

}  // namespace
}  // namespace sr

extern "C" int sr_add_norm_grad(const sr_norm_grad_rows *rows, void *workspace, size_t workspace_bytes, void *stream) {
    return sr::add_norm_grad(rows, workspace, workspace_bytes, (hipStream_t)stream);
}
