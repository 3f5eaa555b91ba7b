// Dropout from the counter-based generator, with the residual's addition; the mask is never stored.
// The contract of the entry point is stated in include/gqsgd.h.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>

#include "gqsgd.h"
#include "gq_layers.hpp"

namespace gq {

// Units a lane: 4 keep enough in flight in long launches, in short ones more lanes do (bf16, 32 bits: 16384x8192 110, 94 and 90 us with 1, 2
// and 4; 2048x4096 7.7, 7.9, 7.5; 512x4096 3.2, 3.5, 4.0; 1x100003 2.1, 2.5, 3.3).
constexpr int64_t kLongDropout = 1 << 21;

// out = residual + (draw < t ? 0 : x scale).  A lane owns UNITS units, each of eight columns of one row and one (16 bits) or two (32 bits)
// Philox calls.  All loads are asked for before the first draw, so that the calls' arithmetic runs under their latency.
// Bound by memory where draws have 16 bits (16384x8192 bf16 with a residual: 128 us, 6.3 TB/s), by memory and the calls' products
// together with 32 (8192x8192 fp32 without one: 96 us, 5.6 TB/s); a short launch by its latency (100003 fp32: 2.4 us).
template <typename T, bool SHORT, bool RESIDUAL, bool TINY, bool FLAT, int UNITS>
__global__ void __launch_bounds__(kBlock)
dropout_kernel(const T *x, const T *residual, T *out, int64_t rows, uint32_t per_row, int64_t n, Drop drop)
{
    RowUnit at[UNITS];
    Eight<T> v[UNITS], r[UNITS];
#pragma unroll
    for (int k = 0; k < UNITS; k++) {
        at[k] = row_unit<UNITS, FLAT>(blockIdx.x, k, per_row);
        const int64_t c = (int64_t)at[k].unit * 8, row = FLAT ? 0 : at[k].row < rows ? at[k].row : rows - 1;
        ask8<true, TINY>(x + row * n, n, c, v[k]);
        if (RESIDUAL) ask8<true, TINY>(residual + row * n, n, c, r[k]);
    }
#pragma unroll
    for (int k = 0; k < UNITS; k++) {
        if (at[k].row >= rows) return;
        const int64_t c = (int64_t)at[k].unit * 8;
        settle8<TINY>(n, c, v[k]);
        if (RESIDUAL) settle8<TINY>(n, c, r[k]);
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = v[k].f(i);
        const int64_t row = FLAT ? 0 : at[k].row;
        drop8<SHORT>(drop, drop.first + ((uint64_t)row * per_row + at[k].unit) * 8, f);
        if (RESIDUAL) {
#pragma unroll
            for (int i = 0; i < 8; i++) f[i] = r[k].f(i) + f[i];
        }
        store8(out + row * n + c, n - c, f);
    }
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
    const bool flat = n >= 8 && (rows == 1 || n % 8 == 0) && flat_fits(rows * (pitch8(n) / 8));      // whole units a row
    if (flat) n *= rows, rows = 1;
    const int64_t per_row = pitch8(n) / 8, units = rows * per_row;
    const bool four = n >= 8 && units >= kLongDropout;
    const int64_t per_block = (four ? 4 : 1) * kBlock, blocks = (units + per_block - 1) / per_block;
    if (!grid_fits(blocks, kBlock)) return GQ_ERR_INVALID_ARG;
    const Drop d = make_drop(p);
    return with_float_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        auto go = [&](auto shorter, auto with_residual) {
            constexpr bool SHORT = decltype(shorter)::value, RESIDUAL = decltype(with_residual)::value;
            auto kernel = n < 8 ? dropout_kernel<T, SHORT, RESIDUAL, true, false, 1>
                          : flat ? (four ? dropout_kernel<T, SHORT, RESIDUAL, false, true, 4> : dropout_kernel<T, SHORT, RESIDUAL, false, true, 1>)
                                 : (four ? dropout_kernel<T, SHORT, RESIDUAL, false, false, 4> : dropout_kernel<T, SHORT, RESIDUAL, false, false, 1>);
            kernel<<<(unsigned)blocks, kBlock, 0, (hipStream_t)hip_stream>>>((const T *)x, (const T *)residual, (T *)out, rows, (uint32_t)per_row, n, d);
            return launched();
        };
        const std::true_type yes;
        const std::false_type no;
        return short_draws(p) ? (residual ? go(yes, yes) : go(yes, no)) : (residual ? go(no, yes) : go(no, no));
    });
}
