// 4-bit weights under group scales: making them and unfolding them.
// The contract of the entry points is stated in include/gqsgd.h.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>

#include "gqsgd.h"
#include "gq_layers.hpp"

namespace gq {

// w / scale to the nearest integer, ties to even, of the exact quotient: the product with 1 / scale (to 2^-22) rounds to the nearest
// integer q or, next to a border, its neighbour.  w - q scale is exact there (it is a multiple of half an ulp of scale and below scale),
// and says which.  The largest magnitude of the group is 7 scale to within scale's rounding, so 7 is not passed.
__device__ __forceinline__ float code_of_quotient(float w, float scale, float inv)
{
    const float q = __builtin_rintf(w * inv), r = __builtin_fmaf(-q, scale, w);
    const float over = __builtin_fmaf(__builtin_fabsf(r), 2.0f, -scale);      // beyond the border, on it, or short of it
    // q + 0.75 goes to the next integer, q + 0.5 to the even one
    const float by = over > 0.0f ? 0.75f : over == 0.0f ? 0.5f : 0.0f;
    return __builtin_rintf(q + __builtin_copysignf(by, r));
}

template <typename S> struct GroupScale { S stored; float scale, inv; };
template <typename S> __device__ __forceinline__ GroupScale<S> group_scale(uint32_t top_bits)
{
    if (top_bits >= 0x7F800000u) return {(S)__builtin_nanf(""), 0.0f, 0.0f};
    const S stored = (S)(__uint_as_float(top_bits) * (1.0f / 7.0f));
    const float scale = (float)stored;
    if (!(scale > 0x1p-128f)) return {(S)0.0f, 0.0f, 0.0f};                   // 1 / scale is not finite
    return {stored, scale, scale >= 0x1p-120f ? __builtin_amdgcn_rcpf(scale) : 1.0f / scale};   // an ulp does not matter to the codes
}

// Eight codes -7 .. 7 as nibbles, four at a time put together as floats (exact below 2^24) and converted together: a bias of 8 in
// every field keeps the sum non-negative, flipping the fields' top bits takes it out again.
__device__ __forceinline__ uint32_t eight_nibbles(const float *q)
{
    uint32_t half[2];
#pragma unroll
    for (int h = 0; h < 2; h++)
        half[h] = (uint32_t)__builtin_fmaf(q[4 * h + 3], 4096.0f, __builtin_fmaf(q[4 * h + 2], 256.0f, __builtin_fmaf(q[4 * h + 1], 16.0f, q[4 * h] + 34952.0f)));
    return (half[0] | (half[1] << 16)) ^ 0x88888888u;
}

// A lane owns UNITS units, each of eight consecutive columns (16 or 32 bytes of weights, one word of codes), a group is 4, 8 or 16
// neighbouring lanes: the maximum goes round them by DPP within a row of 16 lanes.  Units past the row's last column (a row
// is padded to whole groups of units) hold zeros; those within the padding of the row's codes write them.  Bound by memory, read
// once, written once: 8192x8192 bf16, groups of 128, 32.3 us with unfolding in between, 5.2 TB/s, and
// 38.7 in a loop of its own; fp32, groups of 32, 56.5; 1001x4999 fp32 6.4.
template <typename T, typename S, int GROUP, bool TINY, bool FLAT, int UNITS>
__global__ void __launch_bounds__(kBlock)
group_quantize_kernel(const T *w, int64_t rows, int64_t cols, uint32_t units_per_row, int groups, uint32_t row_words, uint32_t *codes, S *scales)
{
    RowUnit at[UNITS];
    Eight<T> x[UNITS];
#pragma unroll
    for (int k = 0; k < UNITS; k++) {
        at[k] = row_unit<UNITS, FLAT>(blockIdx.x, k, units_per_row);
        ask8<true, TINY>(FLAT ? w : w + (at[k].row < rows ? at[k].row : rows - 1) * cols, cols, (int64_t)at[k].unit * 8, x[k]);
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
            float q[8];
#pragma unroll
            for (int i = 0; i < 8; i++) q[i] = code_of_quotient(v[i], gs.scale, gs.inv);
            word = eight_nibbles(q);
        }
        if (at[k].row < rows) {
            const int64_t row = FLAT ? 0 : at[k].row;
            if (FLAT || at[k].unit < row_words) __builtin_nontemporal_store(word, codes + row * row_words + at[k].unit);
            if (at[k].unit % (GROUP / 8) == 0) scales[row * groups + at[k].unit / (GROUP / 8)] = gs.stored;
        }
    }
}

// value = code scale.  A lane owns UNITS units of 16 bytes of values, eight columns and a word of codes, or four (binary32) and half a word, so
// that a wave's stores lie next to each other.  Bound by its writes: 8192x8192 bf16 29.3 us, 5.8 TB/s,
// fp32 57 us, 5.3 TB/s (with eight columns a lane 76); 8001x4999 fp32 45.5 (53.8), 1001x4999 7.8 (7.7).
template <typename T, typename S, bool FLAT, int UNITS>
__global__ void __launch_bounds__(kBlock)
group_dequantize_kernel(const uint32_t *codes, const S *scales, int64_t rows, int64_t cols, uint32_t units_per_row, int group_shift, int groups,
                        uint32_t row_words, T *out)
{
    constexpr int kPer = 16 / sizeof(T), kShift = kPer == 8 ? 3 : 2;
    RowUnit at[UNITS];
    uint32_t word[UNITS];
    S scale[UNITS];
#pragma unroll
    for (int k = 0; k < UNITS; k++) {
        at[k] = row_unit<UNITS, FLAT>(blockIdx.x, k, units_per_row);
        const int64_t row = FLAT ? 0 : at[k].row < rows ? at[k].row : rows - 1;
        const uint32_t unit = FLAT ? min(at[k].unit, units_per_row - 1) : at[k].unit;
        word[k] = __builtin_nontemporal_load(codes + row * row_words + (unit >> (3 - kShift)));
        scale[k] = scales[row * groups + (unit >> (group_shift - kShift))];
    }
#pragma unroll
    for (int k = 0; k < UNITS; k++) {
        if (at[k].row >= rows) return;
        const uint32_t w = kPer == 8 ? word[k] : word[k] >> 16 * (at[k].unit & 1);
        float v[8];
#pragma unroll
        for (int i = 0; i < kPer; i++) v[i] = (float)((int)(w << (28 - 4 * i)) >> 28) * (float)scale[k];
        T *to = out + (FLAT ? 0 : at[k].row) * cols + (int64_t)at[k].unit * kPer;
        const int64_t left = cols - (int64_t)at[k].unit * kPer;
        if constexpr (kPer == 8) {
            store8(to, left, v);
        } else if (left >= 4) {
            typename Chunk<4>::type c;
#pragma unroll
            for (int i = 0; i < 4; i++) c[i] = __float_as_uint(v[i]);
            *reinterpret_cast<typename Chunk<4>::type *>(to) = c;
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (i < left) to[i] = v[i];
        }
    }
}

}  // namespace gq

using namespace gq;

// Units a lane: more keep more in flight in long launches, in short ones more lanes do.  us with 1, 2 and 4, groups of 128:
//   quantise  bf16  2048x4096 6.4, 6.7, 7.3   4096x4096 10.6, 11.3, 11.2   8192x8192 36.0, 35.6, 34.6   8001x8191 43.4, 40.3, 38.0
//             fp32  2048x4096 9.1, 8.8, 9.3   4096x4096 15.2, 15.3, 15.5   8192x8192 53.5, 54.4, 54.8   8001x8191 52.6, 53.0, 55.2
//   unfold    bf16  512x4096 2.5, 2.6, 2.9    2048x4096 5.4, 4.4, 4.3      8192x8192 34.8, 30.2, 30.8   8001x8191 37.4, 34.1, 34.3
//             fp32  512x4096 3.4, 3.4, 3.5    2048x4096 10.6, 9.5, 8.4     8192x8192 63.5, 57.3, 55.0   8001x8191 71.0, 60.6, 66.1
constexpr int64_t kLongQuantize = 1 << 21, kLongUnfold = 1 << 20;
// rows of whole groups: codes and scales of a row end where the next one's begin, the matrix is one row
static bool is_flat(int64_t rows, int64_t cols, int group) { return cols % group == 0 && flat_fits(rows * (cols / 4)); }

extern "C" {

int64_t gq_w4_row_bytes(int64_t cols) { return cols < 0 || cols > kMaxWeightCols ? 0 : (cols + 31) / 32 * 16; }

gq_status gq_group_quantize(const void *w, int64_t rows, int64_t cols, gq_dtype dtype, int group, void *codes_out, void *scales_out,
                            gq_dtype scale_dtype, void *hip_stream)
{
    const gq_status st = check_weights(rows, cols, group, scale_dtype);
    if (st != GQ_OK) return st;
    if (!float_type(dtype)) return GQ_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return GQ_OK;
    if (!aligned(w, 16) || !aligned(codes_out, 16) || !aligned(scales_out, 16)) return GQ_ERR_INVALID_ARG;
    const bool flat = is_flat(rows, cols, group);
    if (flat) cols *= rows, rows = 1;
    // whole groups of units, whole words of codes
    const int64_t row_words = (cols + 31) / 32 * 4, per_row = ((cols + group - 1) / group * group) / 8, units = rows * per_row;
    const bool four = cols >= 8 && dtype != GQ_F32 && units >= kLongQuantize;
    const int64_t groups = (cols + group - 1) / group, per_block = (four ? 4 : 1) * kBlock;
    return with_float_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return with_scale_type(scale_dtype, [&](auto s) {
            typedef decltype(s) S;
            auto of_group = [&](auto g) {
                constexpr int GROUP = decltype(g)::value;
                constexpr int kFour = sizeof(T) == 2 ? 4 : 1;
                return cols < 8 ? group_quantize_kernel<T, S, GROUP, true, false, 1>
                       : flat ? (four ? group_quantize_kernel<T, S, GROUP, false, true, kFour> : group_quantize_kernel<T, S, GROUP, false, true, 1>)
                              : (four ? group_quantize_kernel<T, S, GROUP, false, false, kFour> : group_quantize_kernel<T, S, GROUP, false, false, 1>);
            };
            auto kernel = group == 32 ? of_group(std::integral_constant<int, 32>())
                                      : group == 64 ? of_group(std::integral_constant<int, 64>()) : of_group(std::integral_constant<int, 128>());
            return in_launches(rows, per_row, four ? 4 : 1, [&](int64_t first, int64_t count) {
                kernel<<<(unsigned)((count * per_row + per_block - 1) / per_block), kBlock, 0, (hipStream_t)hip_stream>>>(
                    (const T *)w + first * cols, count, cols, (uint32_t)per_row, (int)groups, (uint32_t)row_words, (uint32_t *)codes_out + first * row_words,
                    (S *)scales_out + first * groups);
                return launched();
            });
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
    const bool flat = is_flat(rows, cols, group);
    if (flat) cols *= rows, rows = 1;
    const int64_t row_words = (cols + 31) / 32 * 4, per = 16 / (int64_t)dtype_size(dtype), per_row = (cols + per - 1) / per, units = rows * per_row;
    const bool four = cols >= 8 && units >= kLongUnfold;
    const int64_t per_block = (four ? 4 : 1) * kBlock, blocks = (units + per_block - 1) / per_block;
    if (!grid_fits(blocks, kBlock)) return GQ_ERR_INVALID_ARG;
    return with_float_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return with_scale_type(scale_dtype, [&](auto s) {
            typedef decltype(s) S;
            auto kernel = flat ? (four ? group_dequantize_kernel<T, S, true, 4> : group_dequantize_kernel<T, S, true, 1>)
                               : (four ? group_dequantize_kernel<T, S, false, 4> : group_dequantize_kernel<T, S, false, 1>);
            kernel<<<(unsigned)blocks, kBlock, 0, (hipStream_t)hip_stream>>>(
                (const uint32_t *)codes, (const S *)scales, rows, cols, (uint32_t)per_row, group == 32 ? 5 : group == 64 ? 6 : 7,
                (int)((cols + group - 1) / group), (uint32_t)row_words, (T *)out);
            return launched();
        });
    });
}

}  // extern "C"
