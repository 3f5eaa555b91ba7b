// What the layers around the gradient exchange share (dropout.hip, rms_norm.hip, weights.hip): element types, eight
// consecutive columns at any alignment, the dropout decision, and the host's checks.
// Internal to the library; the public surface is include/gqsgd.h.
#pragma once
#include "gq_device.hpp"
#include "gq_host.hpp"

#include <math.h>
#include <string.h>

namespace gq {

typedef __bf16 bf16;
typedef _Float16 f16;

// A row of n columns of which eight consecutive ones are a lane's unit.  Rows may begin at any multiple of the element's size:
// the hardware loads and stores 16 bytes at such addresses, so odd row lengths need no path of their own, only a guarded
// last unit.
template <typename T> struct Eight { T e[8]; };

template <typename T> __device__ __forceinline__ void load8(const T *p, int valid, float *v)
{
    Eight<T> t;
    if (valid >= 8) {
        __builtin_memcpy(&t, p, sizeof(t));
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) t.e[i] = i < valid ? p[i] : (T)0.0f;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = (float)t.e[i];
}

template <typename T> __device__ __forceinline__ void store8(T *p, int valid, const float *v)
{
    Eight<T> t;
#pragma unroll
    for (int i = 0; i < 8; i++) t.e[i] = (T)v[i];                      // to nearest even
    if (valid >= 8) {
        __builtin_memcpy(p, &t, sizeof(t));
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < valid) p[i] = t.e[i];
    }
}

// Row and unit within it of a workgroup's lane, where rows have `per_row` units: one 64-bit division a workgroup, on the scalar
// unit, and a 32-bit one a lane.
struct RowUnit { int64_t row; uint32_t unit; };
__device__ __forceinline__ RowUnit row_unit(uint32_t block, uint32_t per_row)
{
    const uint64_t first = (uint64_t)block * kBlock, row = first / per_row;
    const uint32_t at = (uint32_t)(first - row * per_row) + threadIdx.x;           // below 2^28 + 256 for every matrix that fits
    const uint32_t more = at / per_row;
    return {(int64_t)row + more, at - more * per_row};
}

// The dropout decision of gq_dropout_params, as the kernels take it.
struct Drop {
    uint32_t k0, k1, worker;
    uint32_t threshold;   // dropped iff the draw (32 bits, or 16 moved to the top of 32) is below it
    uint64_t first;       // index_base
    float scale;          // of what is kept
};

// v[0..7], the elements g .. g + 7 of the stream (g a multiple of 4, of 8 with short draws), after dropout
template <bool SHORT> __device__ __forceinline__ void drop8(const Drop &d, uint64_t g, float *v)
{
    uint32_t r[8];
    if (SHORT) {
        const uint64_t call = g >> 3;
        const Words4 w = philox4x32_10<false>((uint32_t)call, (uint32_t)(call >> 32), d.worker, 3u, d.k0, d.k1);
#pragma unroll
        for (int i = 0; i < 8; i++) r[i] = short_draw(w.w + (i & 4) / 2, i & 3);
    } else {
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const uint64_t call = (g >> 2) + (uint64_t)h;
            const Words4 w = philox4x32_10<false>((uint32_t)call, (uint32_t)(call >> 32), d.worker, 3u, d.k0, d.k1);
#pragma unroll
            for (int i = 0; i < 4; i++) r[4 * h + i] = w.w[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = r[i] >= d.threshold ? v[i] * d.scale : 0.0f;
}

// ---- host ----------------------------------------------------------------------------------------------------------

static inline int64_t pitch8(int64_t n) { return (n + 7) / 8 * 8; }
static inline size_t dtype_size(int t) { return t == GQ_F32 ? 4 : t == GQ_BF16 || t == GQ_F16 ? 2 : 1; }
static inline bool float_type(int t) { return t == GQ_F32 || t == GQ_BF16 || t == GQ_F16; }
// as far as one launch reaches: 2^35 elements, rows and columns within 31 bits
static inline bool matrix_fits(int64_t rows, int64_t n)
{
    return rows >= 0 && n >= 0 && rows <= 0x7FFFFFFF && n <= 0x7FFFFFF0 && (n == 0 || rows <= ((int64_t)1 << 35) / pitch8(n));
}
static inline bool aligned_or_null(const void *p, size_t a) { return p == nullptr || aligned(p, a); }

// rows, n: of a matrix that fits
static inline gq_status check_drop(const gq_dropout_params *p, int64_t rows, int64_t n)
{
    if (!p) return GQ_ERR_INVALID_ARG;
    if (!(p->p >= 0.0 && p->p < 1.0)) return GQ_ERR_INVALID_ARG;
    if (p->rng_bits != 0 && p->rng_bits != 16 && p->rng_bits != 32) return GQ_ERR_INVALID_ARG;
    if (p->index_base < 0 || p->index_base % (p->rng_bits == 16 ? 8 : 4) != 0) return GQ_ERR_INVALID_ARG;
    if (p->index_base > INT64_MAX - rows * pitch8(n)) return GQ_ERR_INVALID_ARG;
    return GQ_OK;
}
static inline bool short_draws(const gq_dropout_params *p) { return p->rng_bits == 16; }
static inline Drop make_drop(const gq_dropout_params *p)
{
    const int bits = short_draws(p) ? 16 : 32;
    const double all = (double)((int64_t)1 << bits), most = all - 1.0;
    double t = nearbyint(p->p * all);                                   // exact product; ties to even in the default mode
    t = t < most ? t : most;
    return Drop{(uint32_t)p->seed, (uint32_t)(p->seed >> 32), p->worker, (uint32_t)t << (32 - bits), (uint64_t)p->index_base,
                (float)(all / (all - t))};
}

// f(T{}) with the element type that a gq_dtype stands for
template <typename F> static inline gq_status with_float_type(int t, F &&f)
{
    return t == GQ_F32 ? f(float()) : t == GQ_BF16 ? f(bf16()) : f(f16());
}

// 4-bit weights
static inline gq_status check_weights(int64_t rows, int64_t cols, int group, int scale_dtype)
{
    if (!matrix_fits(rows, cols) || rows > (1 << 30) || cols > (1 << 24) || (group != 32 && group != 64 && group != 128)) return GQ_ERR_INVALID_ARG;
    return scale_dtype == GQ_F32 || scale_dtype == GQ_BF16 ? GQ_OK : GQ_ERR_INVALID_ARG;
}
template <typename F> static inline gq_status with_scale_type(int t, F &&f) { return t == GQ_F32 ? f(float()) : f(bf16()); }

}  // namespace gq
