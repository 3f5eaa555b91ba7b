// 4-bit weights under group scales: making them and unfolding them.
// The contract of the entry points is stated in include/gqsgd.h.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>

#include "gqsgd.h"
#include "gq_layers.hpp"

namespace gq {

// w / scale to the nearest integer, ties to even, of the exact quotient: the product with fl32(1 / scale) is off by less than
// 2^-22 and so rounds to the nearest integer or, next to a border, its neighbour.  w - q scale is exact there (it is a multiple of
// half an ulp of scale and below scale), and says which.
__device__ __forceinline__ float code_of_quotient(float w, float scale, float inv)
{
    float q = __builtin_rintf(w * inv);
    const float r = __builtin_fmaf(-q, scale, w), twice = 2.0f * __builtin_fabsf(r);
    const bool odd = (int)q & 1;
    if (twice > scale || (twice == scale && odd)) q += __builtin_copysignf(1.0f, r);
    return __builtin_amdgcn_fmed3f(q, -7.0f, 7.0f);
}

template <typename S> struct GroupScale { S stored; float scale, inv; };
template <typename S> __device__ __forceinline__ GroupScale<S> group_scale(uint32_t top_bits)
{
    if (top_bits >= 0x7F800000u) return {(S)__builtin_nanf(""), 0.0f, 0.0f};
    const S stored = (S)(__uint_as_float(top_bits) / 7.0f);
    const float scale = (float)stored, inv = 1.0f / scale;
    if (!(inv <= 3.402823466e+38f)) return {(S)0.0f, 0.0f, 0.0f};
    return {stored, scale, inv};
}

// A lane owns a unit of eight consecutive columns (16 or 32 bytes of weights, one word of codes), a group is 4, 8 or 16
// neighbouring lanes: the maximum goes round them by DPP within a row of 16 lanes.  Units past the row's last column (a row
// is padded to whole groups of units) hold zeros; those within the padding of the row's codes write them.  Bound by memory: read
// once, written once.
template <typename T, typename S, int GROUP>
__global__ void __launch_bounds__(kBlock)
group_quantize_kernel(const T *w, int64_t units, int64_t cols, uint32_t units_per_row, int groups, uint32_t row_words, uint32_t *codes, S *scales)
{
    const int64_t u = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    const RowUnit at = row_unit(blockIdx.x, units_per_row);
    const int64_t left = cols - (int64_t)at.unit * 8;
    const int valid = u >= units || left <= 0 ? 0 : left < 8 ? (int)left : 8;
    float v[8];
    if (valid > 0) {
        load8(w + at.row * cols + (int64_t)at.unit * 8, valid, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = 0.0f;
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    m = max(m, dpp32<kDppQuadXor1>(m));
    m = max(m, dpp32<kDppQuadXor2>(m));
    if (GROUP >= 64) m = max(m, dpp32<kDppHalfMirror>(m));
    if (GROUP >= 128) m = max(m, dpp32<kDppMirror>(m));
    const GroupScale<S> gs = group_scale<S>(m);
    if (u >= units) return;
    uint32_t word = 0;
    if (gs.inv != 0.0f) {
#pragma unroll
        for (int i = 0; i < 8; i++) word |= ((uint32_t)(int)code_of_quotient(v[i], gs.scale, gs.inv) & 15u) << (4 * i);
    }
    if (at.unit < row_words) codes[at.row * row_words + at.unit] = word;
    if (at.unit % (GROUP / 8) == 0) scales[at.row * groups + at.unit / (GROUP / 8)] = gs.stored;
}

// A lane per eight columns.
template <typename T, typename S>
__global__ void __launch_bounds__(kBlock)
group_dequantize_kernel(const uint32_t *codes, const S *scales, int64_t units, int64_t cols, uint32_t units_per_row, int group_shift, int groups,
                        uint32_t row_words, T *out)
{
    const int64_t u = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (u >= units) return;
    const RowUnit at = row_unit(blockIdx.x, units_per_row);
    const int64_t c = (int64_t)at.unit * 8;
    const uint32_t word = codes[at.row * row_words + at.unit];
    const float scale = (float)scales[at.row * groups + (c >> group_shift)];
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = (float)((int)(word << (28 - 4 * i)) >> 28) * scale;
    store8(out + at.row * cols + c, (int)(cols - c < 8 ? cols - c : 8), v);
}

}  // namespace gq

using namespace gq;

extern "C" {

int64_t gq_w4_row_bytes(int64_t cols) { return cols < 0 || !matrix_fits(1, cols) ? 0 : (cols + 31) / 32 * 16; }

gq_status gq_group_quantize(const void *w, int64_t rows, int64_t cols, gq_dtype dtype, int group, void *codes_out, void *scales_out,
                            gq_dtype scale_dtype, void *hip_stream)
{
    const gq_status st = check_weights(rows, cols, group, scale_dtype);
    if (st != GQ_OK) return st;
    if (!float_type(dtype)) return GQ_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return GQ_OK;
    if (!aligned(w, 16) || !aligned(codes_out, 16) || !aligned(scales_out, 16)) return GQ_ERR_INVALID_ARG;
    // whole groups of units, whole words of codes
    const int64_t per_row = ((cols + group - 1) / group * group) / 8, units = rows * per_row, blocks = (units + kBlock - 1) / kBlock;
    if (!grid_fits(blocks, kBlock)) return GQ_ERR_INVALID_ARG;
    return with_float_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return with_scale_type(scale_dtype, [&](auto s) {
            typedef decltype(s) S;
            auto kernel = group == 32 ? group_quantize_kernel<T, S, 32> : group == 64 ? group_quantize_kernel<T, S, 64> : group_quantize_kernel<T, S, 128>;
            kernel<<<(unsigned)blocks, kBlock, 0, (hipStream_t)hip_stream>>>((const T *)w, units, cols, (uint32_t)per_row, (int)((cols + group - 1) / group),
                                                                           (uint32_t)(gq_w4_row_bytes(cols) / 4), (uint32_t *)codes_out, (S *)scales_out);
            return launched();
        });
    });
}

gq_status gq_group_dequantize(const void *codes, const void *scales, gq_dtype scale_dtype, int64_t rows, int64_t cols, int group, void *out,
                              gq_dtype dtype, void *hip_stream)
{
    const gq_status st = check_weights(rows, cols, group, scale_dtype);
    if (st != GQ_OK) return st;
    if (!float_type(dtype)) return GQ_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return GQ_OK;
    if (!aligned(codes, 16) || !aligned(scales, 16) || !aligned(out, 16)) return GQ_ERR_INVALID_ARG;
    const int64_t per_row = (cols + 7) / 8, units = rows * per_row, blocks = (units + kBlock - 1) / kBlock;
    if (!grid_fits(blocks, kBlock)) return GQ_ERR_INVALID_ARG;
    return with_float_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return with_scale_type(scale_dtype, [&](auto s) {
            typedef decltype(s) S;
            group_dequantize_kernel<T, S><<<(unsigned)blocks, kBlock, 0, (hipStream_t)hip_stream>>>(
                (const uint32_t *)codes, (const S *)scales, units, cols, (uint32_t)per_row, group == 32 ? 5 : group == 64 ? 6 : 7,
                (int)((cols + group - 1) / group), (uint32_t)(gq_w4_row_bytes(cols) / 4), (T *)out);
            return launched();
        });
    });
}

}  // extern "C"
