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

// A lane owns UNITS units, each of eight consecutive columns (16 or 32 bytes of weights, one word of codes), a group is 4, 8 or 16
// neighbouring lanes: the maximum goes round them by DPP within a row of 16 lanes.  Units past the row's last column (a row
// is padded to whole groups of units) hold zeros; those within the padding of the row's codes write them.  Bound by memory: read
// once, written once.
template <typename T, typename S, int GROUP, bool TINY, int UNITS>
__global__ void __launch_bounds__(kBlock)
group_quantize_kernel(const T *w, int64_t rows, int64_t cols, uint32_t units_per_row, int groups, uint32_t row_words, uint32_t *codes, S *scales)
{
    RowUnit at[UNITS];
    Eight<T> x[UNITS];
#pragma unroll
    for (int k = 0; k < UNITS; k++) {
        at[k] = row_unit<UNITS>(blockIdx.x, k, units_per_row);
        ask8<true, TINY>(w + (at[k].row < rows ? at[k].row : rows - 1) * cols, cols, (int64_t)at[k].unit * 8, x[k]);
    }
#pragma unroll
    for (int k = 0; k < UNITS; k++) {
        settle8<TINY>(cols, (int64_t)at[k].unit * 8, x[k]);
        float v[8];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            v[i] = x[k].f(i);
            m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
        }
        m = max(m, dpp32<kDppQuadXor1>(m));
        m = max(m, dpp32<kDppQuadXor2>(m));
        if (GROUP >= 64) m = max(m, dpp32<kDppHalfMirror>(m));
        if (GROUP >= 128) m = max(m, dpp32<kDppMirror>(m));
        const GroupScale<S> gs = group_scale<S>(m);
        uint32_t word = 0;
        if (gs.inv != 0.0f) {
#pragma unroll
            for (int i = 0; i < 8; i++) word |= ((uint32_t)(int)code_of_quotient(v[i], gs.scale, gs.inv) & 15u) << (4 * i);
        }
        if (at[k].row < rows) {
            if (at[k].unit < row_words) __builtin_nontemporal_store(word, codes + at[k].row * row_words + at[k].unit);
            if (at[k].unit % (GROUP / 8) == 0) scales[at[k].row * groups + at[k].unit / (GROUP / 8)] = gs.stored;
        }
    }
}

// The same units.
template <typename T, typename S, int UNITS>
__global__ void __launch_bounds__(kBlock)
group_dequantize_kernel(const uint32_t *codes, const S *scales, int64_t rows, int64_t cols, uint32_t units_per_row, int group_shift, int groups,
                        uint32_t row_words, T *out)
{
    RowUnit at[UNITS];
    uint32_t word[UNITS];
    S scale[UNITS];
#pragma unroll
    for (int k = 0; k < UNITS; k++) {
        at[k] = row_unit<UNITS>(blockIdx.x, k, units_per_row);
        const int64_t row = at[k].row < rows ? at[k].row : rows - 1;
        word[k] = __builtin_nontemporal_load(codes + row * row_words + at[k].unit);
        scale[k] = scales[row * groups + (at[k].unit >> (group_shift - 3))];
    }
#pragma unroll
    for (int k = 0; k < UNITS; k++) {
        if (at[k].row >= rows) return;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = (float)((int)(word[k] << (28 - 4 * i)) >> 28) * (float)scale[k];
        store8(out + at[k].row * cols + (int64_t)at[k].unit * 8, cols - (int64_t)at[k].unit * 8, v);
    }
}

}  // namespace gq

using namespace gq;

// Units a lane: 4 keep enough in flight in long launches, in short ones more lanes do (quantise 8192x8192 bf16: 47.1, 44.9 and 43.7 us
// with 1, 2 and 4, unfold 35.1, 33.5, 32.0; 2048x4096: 8.1, 7.9, 9.4 and 5.8, 5.9, 6.7; 128x4096: 3.0, 3.8, 5.6 and 1.9, 2.1, 2.5).
constexpr int64_t kLongWeights = 1 << 21;
static bool long_launch(int64_t units, int64_t cols) { return cols >= 8 && units >= kLongWeights; }

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
    const int64_t per_row = ((cols + group - 1) / group * group) / 8, units = rows * per_row, per_block = (int64_t)(long_launch(units, cols) ? 4 : 1) * kBlock, blocks = (units + per_block - 1) / per_block;
    if (!grid_fits(blocks, kBlock)) return GQ_ERR_INVALID_ARG;
    return with_float_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return with_scale_type(scale_dtype, [&](auto s) {
            typedef decltype(s) S;
            auto of_group = [&](auto g) {
                constexpr int GROUP = decltype(g)::value;
                return cols < 8 ? group_quantize_kernel<T, S, GROUP, true, 1>
                                : long_launch(units, cols) ? group_quantize_kernel<T, S, GROUP, false, 4> : group_quantize_kernel<T, S, GROUP, false, 1>;
            };
            auto kernel = group == 32 ? of_group(std::integral_constant<int, 32>())
                                      : group == 64 ? of_group(std::integral_constant<int, 64>()) : of_group(std::integral_constant<int, 128>());
            kernel<<<(unsigned)blocks, kBlock, 0, (hipStream_t)hip_stream>>>((const T *)w, rows, cols, (uint32_t)per_row, (int)((cols + group - 1) / group),
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
    const int64_t per_row = (cols + 7) / 8, units = rows * per_row, per_block = (int64_t)(long_launch(units, cols) ? 4 : 1) * kBlock, blocks = (units + per_block - 1) / per_block;
    if (!grid_fits(blocks, kBlock)) return GQ_ERR_INVALID_ARG;
    return with_float_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return with_scale_type(scale_dtype, [&](auto s) {
            typedef decltype(s) S;
            auto kernel = long_launch(units, cols) ? group_dequantize_kernel<T, S, 4> : group_dequantize_kernel<T, S, 1>;
            kernel<<<(unsigned)blocks, kBlock, 0, (hipStream_t)hip_stream>>>(
                (const uint32_t *)codes, (const S *)scales, rows, cols, (uint32_t)per_row, group == 32 ? 5 : group == 64 ? 6 : 7,
                (int)((cols + group - 1) / group), (uint32_t)(gq_w4_row_bytes(cols) / 4), (T *)out);
            return launched();
        });
    });
}

}  // extern "C"
