// Dropout from the counter-based generator, with the residual's addition; the mask is never stored.
// The contract of the entry point is stated in include/gqsgd.h.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>

#include "gqsgd.h"
#include "gq_layers.hpp"

namespace gq {

// A lane owns a unit: eight columns of one row, one (16 bits) or two (32 bits) Philox calls.
template <typename T, bool SHORT>
__global__ void __launch_bounds__(kBlock)
dropout_kernel(const T *x, const T *residual, T *out, int64_t units, uint32_t per_row, int64_t n, Drop drop)
{
    const int64_t u = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (u >= units) return;
    const RowUnit ru = row_unit(blockIdx.x, per_row);
    const int64_t at = ru.row * n + (int64_t)ru.unit * 8;
    const int64_t left = n - (int64_t)ru.unit * 8;
    const int valid = left < 8 ? (int)left : 8;
    float v[8];
    load8(x + at, valid, v);
    drop8<SHORT>(drop, drop.first + (uint64_t)u * 8, v);
    if (residual) {
        float r[8];
        load8(residual + at, valid, r);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = r[i] + v[i];
    }
    store8(out + at, valid, v);
}

}  // namespace gq

using namespace gq;

extern "C" gq_status gq_dropout(const void *x, const void *residual, int64_t rows, int64_t n, gq_dtype dtype,
                                const gq_dropout_params *p, void *out, void *hip_stream)
{
    if (!float_type(dtype) || !matrix_fits(rows, n)) return GQ_ERR_INVALID_ARG;
    const gq_status st = check_drop(p, rows, n);
    if (st != GQ_OK) return st;
    if (rows == 0 || n == 0) return GQ_OK;
    if (!aligned(x, 16) || !aligned(out, 16) || !aligned_or_null(residual, 16)) return GQ_ERR_INVALID_ARG;
    const int64_t per_row = pitch8(n) / 8, units = rows * per_row, blocks = (units + kBlock - 1) / kBlock;
    if (!grid_fits(blocks, kBlock)) return GQ_ERR_INVALID_ARG;
    const Drop d = make_drop(p);
    return with_float_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        auto kernel = short_draws(p) ? dropout_kernel<T, true> : dropout_kernel<T, false>;
        kernel<<<(unsigned)blocks, kBlock, 0, (hipStream_t)hip_stream>>>((const T *)x, (const T *)residual, (T *)out, units,
                                                                       (uint32_t)per_row, n, d);
        return launched();
    });
}
