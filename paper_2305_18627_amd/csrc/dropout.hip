// Dropout from the counter-based generator, with the residual's addition; the mask is never stored.
// The contract of the entry point is stated in include/gqsgd.h.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>

#include "gqsgd.h"
#include "gq_layers.hpp"

namespace gq {

// out = residual + (draw < t ? 0 : x scale).  A lane owns a unit of eight columns of one row and one (16 bits) or two (32 bits) Philox calls.
// Both loads are asked for before the first draw, so that the calls' arithmetic runs under their latency.  Several units a lane keep
// more in flight and are no faster, us with 1, 2 and 4: 16384x8192 bf16 with a residual 126, 132, 131, 8192x8192 bf16 43, 47, 48, fp32 95, 96, 97,
// 4096x4096 bf16 12.2, 14.9, 14.2, 512x4096 3.0, 3.8, 4.1; only fp32 in odd rows without a residual gains a little (8001x8191 107, 103, 105).
// Bound by memory: 16384x8192 bf16 with a residual 122 us, 6.6 TB/s, 8192x8192 fp32 without one 94, 5.7; a short launch by its latency
// (100003 fp32: 2.0 us).
template <typename T, bool SHORT, bool RESIDUAL, bool TINY, bool FLAT>
__global__ void __launch_bounds__(kBlock)
dropout_kernel(const T *x, const T *residual, T *out, int64_t rows, uint32_t per_row, int64_t n, Drop drop)
{
    const RowUnit at = row_unit<1, FLAT>(blockIdx.x, 0, per_row);
    const int64_t row = FLAT ? 0 : at.row < rows ? at.row : rows - 1, c = (int64_t)at.unit * 8;
    Eight<T> v, r;
    ask8<true, TINY>(x + row * n, n, c, v);
    if (RESIDUAL) ask8<true, TINY>(residual + row * n, n, c, r);
    if (at.row >= rows) return;                                       // not before the loads, which would wait for it
    uint32_t draw[8];
    draws8<SHORT>(drop, drop.first + ((uint64_t)row * per_row + at.unit) * 8, draw);
    __builtin_amdgcn_sched_barrier(0);                                // no wait for the loads above this
    settle8<TINY>(n, c, v);
    if (RESIDUAL) settle8<TINY>(n, c, r);
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        f[i] = dropped(drop, draw[i], v.f(i));
        if (RESIDUAL) f[i] = r.f(i) + f[i];
    }
    store8(out + row * n + c, n - c, f);
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
    const int64_t per_row = pitch8(n) / 8;
    const Drop whole = make_drop(p);
    return with_float_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        auto go = [&](auto shorter, auto with_residual) {
            constexpr bool SHORT = decltype(shorter)::value, RESIDUAL = decltype(with_residual)::value;
            auto kernel = n < 8 ? dropout_kernel<T, SHORT, RESIDUAL, true, false>
                          : flat ? dropout_kernel<T, SHORT, RESIDUAL, false, true> : dropout_kernel<T, SHORT, RESIDUAL, false, false>;
            return in_launches(rows, per_row, 1, [&](int64_t first, int64_t count) {
                Drop d = whole;
                d.first += (uint64_t)first * per_row * 8;
                kernel<<<(unsigned)((count * per_row + kBlock - 1) / kBlock), kBlock, 0, (hipStream_t)hip_stream>>>(
                    (const T *)x + first * n, RESIDUAL ? (const T *)residual + first * n : nullptr, (T *)out + first * n, count, (uint32_t)per_row, n, d);
                return launched();
            });
        };
        const std::true_type yes;
        const std::false_type no;
        return short_draws(p) ? (residual ? go(yes, yes) : go(yes, no)) : (residual ? go(no, yes) : go(no, no));
    });
}
