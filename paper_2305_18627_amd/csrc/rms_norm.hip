// Root-mean-square norm with the residual's addition, outputs in the input's type or in 8 bits, and its backward pass.
// The contract of the entry points is stated in include/gqsgd.h.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>

#include "gqsgd.h"
#include "gq_layers.hpp"

namespace gq {

constexpr int kNormBlock = 256;

// the sum over a workgroup, the same for all its lanes
__device__ __forceinline__ double block_sum(double v, double *lds)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
    for (unsigned i = 0; i < blockDim.x / 64; i++) s += lds[i];
    return s;
}
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t *lds)
{
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    uint32_t m = 0;
    for (unsigned i = 0; i < blockDim.x / 64; i++) m = max(m, lds[i]);
    return m;
}

struct RowScale { float scale, inv; };
// scale and what codes are multiplied by, for a row whose largest magnitude has the bits `top_bits`
__device__ __forceinline__ RowScale row_scale(uint32_t top_bits, float top)
{
    const float a = __uint_as_float(top_bits);
    if (top_bits >= 0x7F800000u) return {__builtin_nanf(""), 0.0f};
    const float scale = a / top, inv = 1.0f / scale;
    if (!(inv <= 3.402823466e+38f)) return {0.0f, 0.0f};              // a row of zeros, or too small to be scaled
    return {scale, inv};
}

// y inv as a code; a row that is not finite has inv = 0 and gives codes 0 whatever y is
__device__ __forceinline__ float code_of(float y, float inv, float top)
{
    return inv == 0.0f ? 0.0f : __builtin_amdgcn_fmed3f(y * inv, -top, top);
}

// A workgroup per row, the row's h in LDS.
template <typename T, typename W>
__global__ void __launch_bounds__(kNormBlock)
rms_norm_kernel(const T *x, const T *residual, int64_t n, const W *weight, float eps, int with_drop, Drop drop, T *sum_out, void *out,
                int out_dtype, float *scales_out, float *rstd_out)
{
    extern __shared__ float h[];
    __shared__ double sums[kNormBlock / 64];
    __shared__ uint32_t tops[kNormBlock / 64];
    const int64_t row = blockIdx.x, at = row * n;
    const int units = (int)((n + 7) / 8);
    double ss = 0.0;
    for (int u = threadIdx.x; u < units; u += kNormBlock) {
        const int valid = (int)(n - 8 * u < 8 ? n - 8 * u : 8);
        float v[8];
        load8(x + at + 8 * u, valid, v);
        if (with_drop == 32) drop8<false>(drop, drop.first + 8 * ((uint64_t)row * units + u), v);
        if (with_drop == 16) drop8<true>(drop, drop.first + 8 * ((uint64_t)row * units + u), v);
        if (residual) {
            float r[8];
            load8(residual + at + 8 * u, valid, r);
            for (int i = 0; i < 8; i++) v[i] = r[i] + v[i];
        }
        if (sum_out) store8(sum_out + at + 8 * u, valid, v);
        for (int i = 0; i < 8; i++) {
            h[8 * u + i] = v[i];
            ss += (double)v[i] * (double)v[i];
        }
    }
    ss = block_sum(ss, sums);
    const float rstd = (float)(1.0 / sqrt(ss / (double)n + (double)eps));
    if (rstd_out && threadIdx.x == 0) rstd_out[row] = rstd;
    RowScale rs = {1.0f, 1.0f};
    const float top = out_dtype == GQ_I8 ? 127.0f : 448.0f;
    if (scales_out) {
        uint32_t m = 0;
        for (int u = threadIdx.x; u < units; u += kNormBlock)
            for (int i = 0; i < 8; i++)
                if (8 * u + i < n) m = max(m, __float_as_uint((h[8 * u + i] * rstd) * (float)weight[8 * u + i]) & 0x7FFFFFFFu);
        rs = row_scale(block_max(m, tops), top);
        if (threadIdx.x == 0) scales_out[row] = rs.scale;
    }
    for (int u = threadIdx.x; u < units; u += kNormBlock) {
        const int valid = (int)(n - 8 * u < 8 ? n - 8 * u : 8);
        float v[8];
        for (int i = 0; i < 8; i++) v[i] = i < valid ? (h[8 * u + i] * rstd) * (float)weight[8 * u + i] : 0.0f;
        if (!scales_out) {
            store8((T *)out + at + 8 * u, valid, v);
        } else {
            for (int i = 0; i < valid; i++) {
                const float c = code_of(v[i], rs.inv, top);
                if (out_dtype == GQ_I8) ((int8_t *)out)[at + 8 * u + i] = (int8_t)__builtin_rintf(c);
                else ((uint8_t *)out)[at + 8 * u + i] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, c, 0, false);
            }
        }
    }
}

template <typename T, typename W>
__global__ void __launch_bounds__(kNormBlock)
rms_norm_backward_kernel(const T *dy, const T *h, const T *dsum, int64_t n, const W *weight, const float *rstds, int with_drop,
                         Drop drop, T *dres_out, T *dx_out)
{
    __shared__ double sums[kNormBlock / 64];
    const int64_t row = blockIdx.x, at = row * n;
    const int units = (int)((n + 7) / 8);
    const float rstd = rstds[row];
    double s = 0.0;
    for (int64_t c = threadIdx.x; c < n; c += kNormBlock) s += (double)((float)dy[at + c] * (float)weight[c]) * (double)((float)h[at + c] * rstd);
    const float mean = (float)(block_sum(s, sums) / (double)n);
    for (int u = threadIdx.x; u < units; u += kNormBlock) {
        const int valid = (int)(n - 8 * u < 8 ? n - 8 * u : 8);
        float v[8], a[8], b[8];
        load8(dy + at + 8 * u, valid, a);
        load8(h + at + 8 * u, valid, b);
        for (int i = 0; i < 8; i++) v[i] = rstd * (a[i] * (i < valid ? (float)weight[8 * u + i] : 0.0f) - (b[i] * rstd) * mean);
        if (dsum) {
            load8(dsum + at + 8 * u, valid, a);
            for (int i = 0; i < 8; i++) v[i] = a[i] + v[i];
        }
        if (dres_out) store8(dres_out + at + 8 * u, valid, v);
        if (with_drop == 32) drop8<false>(drop, drop.first + 8 * ((uint64_t)row * units + u), v);
        if (with_drop == 16) drop8<true>(drop, drop.first + 8 * ((uint64_t)row * units + u), v);
        store8(dx_out + at + 8 * u, valid, v);
    }
}

constexpr int kWeightParts = 256;      // stretches of rows whose sums are added up by a second kernel

template <typename T>
__global__ void __launch_bounds__(kNormBlock)
weight_partial_kernel(const T *dy, const T *h, int64_t rows, int64_t n, const float *rstds, float *parts)
{
    const int64_t c = (int64_t)blockIdx.x * kNormBlock + threadIdx.x;
    if (c >= n) return;
    const int64_t per = (rows + gridDim.y - 1) / gridDim.y, first = per * blockIdx.y, last = first + per < rows ? first + per : rows;
    float s = 0.0f;
    for (int64_t r = first; r < last; r++) s += (float)dy[r * n + c] * ((float)h[r * n + c] * rstds[r]);
    parts[(int64_t)blockIdx.y * n + c] = s;
}

__global__ void __launch_bounds__(kNormBlock)
weight_sum_kernel(const float *parts, int count, int64_t n, float *dweight)
{
    const int64_t c = (int64_t)blockIdx.x * kNormBlock + threadIdx.x;
    if (c >= n) return;
    float s = 0.0f;
    for (int i = 0; i < count; i++) s += parts[(int64_t)i * n + c];
    dweight[c] = s;
}

static gq_status check_norm(int64_t rows, int64_t n, int dtype, int weight_dtype, const gq_dropout_params *drop)
{
    if (!float_type(dtype) || (weight_dtype != GQ_F32 && weight_dtype != dtype) || !matrix_fits(rows, n)) return GQ_ERR_INVALID_ARG;
    if (drop && check_drop(drop, rows, n) != GQ_OK) return GQ_ERR_INVALID_ARG;
    return n > GQ_RMS_NORM_MAX_N ? GQ_ERR_UNSUPPORTED : GQ_OK;
}
static int draw_bits(const gq_dropout_params *p) { return !p ? 0 : short_draws(p) ? 16 : 32; }

template <typename F> static gq_status with_types(int dtype, int weight_dtype, F &&f)
{
    return with_float_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return weight_dtype == GQ_F32 ? f(t, float()) : f(t, T());
    });
}

static int64_t weight_parts(int64_t rows) { return rows < kWeightParts ? (rows > 0 ? rows : 1) : kWeightParts; }

}  // namespace gq

using namespace gq;

extern "C" {

gq_status gq_rms_norm(const void *x, const void *residual, int64_t rows, int64_t n, gq_dtype dtype, const void *weight,
                      gq_dtype weight_dtype, float eps, const gq_dropout_params *drop, void *sum_out, void *out, gq_dtype out_dtype,
                      float *scales_out, float *rstd_out, void *hip_stream)
{
    const gq_status st = check_norm(rows, n, dtype, weight_dtype, drop);
    if (st != GQ_OK) return st;
    const bool bytes = out_dtype == GQ_I8 || out_dtype == GQ_E4M3;
    if (!(eps > 0.0f && eps <= 3.402823466e+38f) || (!bytes && out_dtype != dtype) || bytes != (scales_out != nullptr)) return GQ_ERR_INVALID_ARG;
    if (rows == 0 || n == 0) return GQ_OK;
    if (!aligned(x, 16) || !aligned(weight, 16) || !aligned(out, 16) || !aligned_or_null(residual, 16) || !aligned_or_null(sum_out, 16) ||
        !aligned_or_null(scales_out, 4) || !aligned_or_null(rstd_out, 4) || out == sum_out) return GQ_ERR_INVALID_ARG;
    if (!grid_fits(rows, kNormBlock)) return GQ_ERR_INVALID_ARG;
    const Drop d = drop ? make_drop(drop) : Drop{};
    return with_types(dtype, weight_dtype, [&](auto t, auto w) {
        typedef decltype(t) T;
        typedef decltype(w) W;
        const unsigned lds = (unsigned)(4 * pitch8(n));
        auto kernel = rms_norm_kernel<T, W>;
        if (hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) return GQ_ERR_DEVICE;
        kernel<<<(unsigned)rows, kNormBlock, lds, (hipStream_t)hip_stream>>>(
            (const T *)x, (const T *)residual, n, (const W *)weight, eps, draw_bits(drop), d, (T *)sum_out, out, out_dtype, scales_out, rstd_out);
        return launched();
    });
}

size_t gq_rms_norm_workspace_bytes(int64_t rows, int64_t n)
{
    if (!matrix_fits(rows, n) || n > GQ_RMS_NORM_MAX_N) return 0;
    return (size_t)(weight_parts(rows) * pitch8(n) * 4);
}

gq_status gq_rms_norm_backward(const void *dy, const void *h, const void *dsum, int64_t rows, int64_t n, gq_dtype dtype,
                               const void *weight, gq_dtype weight_dtype, const float *rstd, const gq_dropout_params *drop, void *dres_out,
                               void *dx_out, float *dweight_out, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const gq_status st = check_norm(rows, n, dtype, weight_dtype, drop);
    if (st != GQ_OK) return st;
    if (!drop && dres_out) return GQ_ERR_INVALID_ARG;
    if (n == 0 || (rows == 0 && !dweight_out)) return GQ_OK;
    if (rows > 0 && (!aligned(dy, 16) || !aligned(h, 16) || !aligned(weight, 16) || !aligned(rstd, 4) || !aligned(dx_out, 16) ||
                     !aligned_or_null(dsum, 16) || !aligned_or_null(dres_out, 16) || dres_out == dx_out)) return GQ_ERR_INVALID_ARG;
    if (!aligned_or_null(dweight_out, 16) || !grid_fits(rows, kNormBlock)) return GQ_ERR_INVALID_ARG;
    if (dweight_out && (!aligned(workspace, 16) || workspace_bytes < gq_rms_norm_workspace_bytes(rows, n))) return GQ_ERR_WORKSPACE;
    const Drop d = drop ? make_drop(drop) : Drop{};
    return with_types(dtype, weight_dtype, [&](auto t, auto w) {
        typedef decltype(t) T;
        typedef decltype(w) W;
        const hipStream_t stream = (hipStream_t)hip_stream;
        if (dweight_out) {                                             // before dx: dx_out may be dy
            const unsigned cols = (unsigned)((n + kNormBlock - 1) / kNormBlock);
            const int parts = (int)weight_parts(rows);
            weight_partial_kernel<T><<<dim3(cols, parts), kNormBlock, 0, stream>>>((const T *)dy, (const T *)h, rows, n, rstd, (float *)workspace);
            weight_sum_kernel<<<cols, kNormBlock, 0, stream>>>((const float *)workspace, parts, n, dweight_out);
        }
        if (rows > 0)
            rms_norm_backward_kernel<T, W><<<(unsigned)rows, kNormBlock, 0, stream>>>((const T *)dy, (const T *)h, (const T *)dsum, n, (const W *)weight, rstd,
                                                                                     draw_bits(drop), d, (T *)dres_out, (T *)dx_out);
        return launched();
    });
}

}  // extern "C"
