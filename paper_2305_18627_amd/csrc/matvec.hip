// Rows of activations times 4-bit weights under group scales.
// The contract of the entry point is stated in include/gqsgd.h.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>

#include "gqsgd.h"
#include "matvec.hpp"

// compiled in files of their own
extern template gq_status gq::matvec<gq::bf16>(const gq::MatvecArgs &, int, int, hipStream_t);
extern template gq_status gq::matvec<gq::f16>(const gq::MatvecArgs &, int, int, hipStream_t);
extern template gq_status gq::matvec<int8_t>(const gq::MatvecArgs &, int, int, hipStream_t);

using namespace gq;

extern "C" gq_status gq_w4_matvec(const void *x, const float *x_scales, int64_t m, gq_dtype x_dtype, const void *codes, const void *scales,
                                  gq_dtype scale_dtype, int64_t rows, int64_t cols, int group, const void *bias, void *y, gq_dtype y_dtype,
                                  void *hip_stream)
{
    const gq_status st = check_weights(rows, cols, group, scale_dtype);
    if (st != GQ_OK) return st;
    if ((x_dtype != GQ_BF16 && x_dtype != GQ_F16 && x_dtype != GQ_I8) || !float_type(y_dtype) || (x_dtype == GQ_I8) != (x_scales != nullptr) ||
        m > (1 << 20) || !matrix_fits(m, cols) || !matrix_fits(m, rows)) return GQ_ERR_INVALID_ARG;
    if (m == 0 || rows == 0) return GQ_OK;
    if (!aligned(y, 16) || !aligned_or_null(bias, 16) || (cols > 0 && (!aligned(x, 16) || !aligned(codes, 16) || !aligned(scales, 16))) ||
        !aligned_or_null(x_scales, 4)) return GQ_ERR_INVALID_ARG;
    const MatvecArgs p = {x, x_scales, (const uint8_t *)codes, scales, bias, y, gq_w4_row_bytes(cols), (int)m, (int)rows, (int)cols,
                          (int)((cols + group - 1) / group), (int)y_dtype, 0};
    const hipStream_t stream = (hipStream_t)hip_stream;
    return x_dtype == GQ_BF16 ? matvec<bf16>(p, group, scale_dtype, stream)
           : x_dtype == GQ_F16 ? matvec<f16>(p, group, scale_dtype, stream) : matvec<int8_t>(p, group, scale_dtype, stream);
}
