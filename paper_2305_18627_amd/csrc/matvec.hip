// Rows of activations times 4-bit weights under group scales, on the matrix cores.
// The contract of the entry point is stated in include/gqsgd.h.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>

#include "gqsgd.h"
#include "gq_layers.hpp"

namespace gq {

// What an activation type brings along.  A lane's eight codes are one word; the instructions take them as eight activations'
// worth of operand B, and x as operand A in the order in which unfolding leaves the codes:
//   16 bits  pairs (i, i + 4): one shift and one v_and_or_b32 put nibbles i and i + 4 of (word ^ 0x88..8) behind the exponent of
//            16.0 of two halves, which are then 16 + (code + 8) = 24 + code exactly.  24 times the sum of x is taken out again by
//            the same instruction with a constant operand of -24.
//   int8     bytes of 16 times a code, even ones (word << 4) and odd ones (word) under 0xF0F0F0F0: three instructions for eight
//            codes; sums are exact integers.
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <typename X> struct Act;
template <typename V, uint32_t ONE, int TOP, uint32_t MINUS> struct Act16 {
    typedef V Operand;
    typedef f32x4 Sum;
    static constexpr bool kMoved = true;
    static constexpr float kUnit = 1.0f;
    static __device__ __forceinline__ Operand unfold(uint32_t w)
    {
        const uint32_t u = w ^ 0x88888888u, mask = 0x000F000Fu << TOP;
        const u32x4 r = {((u << TOP) & mask) | ONE, ((TOP >= 4 ? u << (TOP - 4) : u >> (4 - TOP)) & mask) | ONE,
                         ((TOP >= 8 ? u << (TOP - 8) : u >> (8 - TOP)) & mask) | ONE, ((u >> (12 - TOP)) & mask) | ONE};
        return __builtin_bit_cast(Operand, r);
    }
    static __device__ __forceinline__ Operand minus24() { return __builtin_bit_cast(Operand, u32x4{MINUS, MINUS, MINUS, MINUS}); }
    static constexpr int kOrder[8] = {0, 4, 1, 5, 2, 6, 3, 7};
};
template <> struct Act<bf16> : Act16<bf16x8, 0x41804180u, 3, 0xC1C0C1C0u> {
    static __device__ __forceinline__ Sum product(Operand a, Operand b, Sum c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Act<f16> : Act16<f16x8, 0x4C004C00u, 6, 0xCE00CE00u> {
    static __device__ __forceinline__ Sum product(Operand a, Operand b, Sum c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Act<int8_t> {
    typedef long Operand;
    typedef i32x4 Sum;
    static constexpr bool kMoved = false;
    static constexpr float kUnit = 0.0625f;
    static __device__ __forceinline__ Operand unfold(uint32_t w)
    {
        return __builtin_bit_cast(Operand, u32x2{(w << 4) & 0xF0F0F0F0u, w & 0xF0F0F0F0u});
    }
    static __device__ __forceinline__ Sum product(Operand a, Operand b, Sum c) { return __builtin_amdgcn_mfma_i32_16x16x32_i8(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ Operand minus24() { return 0; }
    static constexpr int kOrder[8] = {0, 2, 4, 6, 1, 3, 5, 7};
};

// d[j] of lane group q (lanes 16 q .. 16 q + 15) becomes d[q] of lane group j
__device__ __forceinline__ void transpose4(uint32_t *d)
{
    const auto a = __builtin_amdgcn_permlane32_swap(d[0], d[2], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(d[1], d[3], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    const auto e = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    d[0] = c[0]; d[1] = c[1]; d[2] = e[0]; d[3] = e[1];
}

struct MatvecArgs {
    const void *x;
    const float *x_scales;
    const uint8_t *codes;
    const void *scales, *bias;
    void *y;
    int64_t row_bytes;
    int m, rows, cols, groups, y_dtype, stage_shift;     // a stage of x in LDS: 2^stage_shift columns
};

// A workgroup of WN x WK waves owns WN * RT * 16 rows of the weights and up to MT * 16 rows of x; the WK waves share out the
// columns, 128 U at a time, and their sums are joined in LDS at the end.  x is staged in LDS, a stage at a time.
template <typename X, typename S, int GROUP, int MT, int RT, int WN, int WK, int U>
__global__ void __launch_bounds__(64 * WN * WK)
w4_matvec_kernel(MatvecArgs p)
{
    typedef Act<X> A;
    typedef typename A::Operand Operand;
    typedef typename A::Sum Sum;
    constexpr int kThreads = 64 * WN * WK, kUnit = 8 * (int)sizeof(X), kSwizzle = 128 / kUnit - 1;
    constexpr int kGroups = 128 / GROUP, kBlocks = GROUP / 32;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wk = wave % WK, wn = wave / WK;
    const int i16 = lane & 15, q = lane >> 4;
    const int first_row = (blockIdx.x * WN + wn) * RT * 16, first_m = blockIdx.y * MT * 16;
    const int m_rows = min(p.m - first_m, MT * 16);
    const X *x = (const X *)p.x + (int64_t)first_m * p.cols;

    const uint8_t *code_row[RT];
    const S *scale_row[RT];
#pragma unroll
    for (int t = 0; t < RT; t++) {
        const int64_t r = min(first_row + 16 * t + i16, p.rows - 1);    // rows past the last one: its codes again, never stored
        code_row[t] = p.codes + r * p.row_bytes;
        scale_row[t] = (const S *)p.scales + r * p.groups;
    }
    struct Fetched { u32x4 w[U][RT]; float s[U][RT][kGroups]; };
    const int last_block = (p.cols + 31) / 32 - 1, steps = (p.cols + 128 * U * WK - 1) / (128 * U * WK);
    auto fetch = [&](int step, Fetched &f) {
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int c = ((step * WK + wk) * U + u) * 128;
            // 16 bytes of codes a lane; past the row's end the last ones again, where x is zero
            const int b = min(c / 32 + q, last_block);
#pragma unroll
            for (int t = 0; t < RT; t++) {
                f.w[u][t] = *reinterpret_cast<const u32x4 *>(code_row[t] + 16 * (int64_t)b);
#pragma unroll
                for (int g = 0; g < kGroups; g++) {
                    const int at = c / GROUP + g;
                    const float s = (float)scale_row[t][min(at, p.groups - 1)];
                    f.s[u][t][g] = at < p.groups ? s : 0.0f;
                }
            }
        }
    };

    const int stage_cols = 1 << p.stage_shift, units_shift = p.stage_shift - 3;
    auto stage = [&](int first_col) {
        for (int u = threadIdx.x; u < (m_rows << units_shift); u += kThreads) {
            const int row = u >> units_shift, unit = u & ((1 << units_shift) - 1), c = first_col + 8 * unit;
            Eight<X> v, o;
            const X *at = x + (int64_t)row * p.cols + c;
            if (c + 8 <= p.cols) {
                __builtin_memcpy(&v, at, sizeof(v));
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++) v.e[i] = c + i < p.cols ? at[i] : (X)0;
            }
#pragma unroll
            for (int i = 0; i < 8; i++) o.e[i] = v.e[A::kOrder[i]];
            *reinterpret_cast<Operand *>(lds + ((row << units_shift) + (unit ^ (row & kSwizzle))) * kUnit) = __builtin_bit_cast(Operand, o);
        }
    };
    int lds_row[MT], lds_mask[MT];
#pragma unroll
    for (int t = 0; t < MT; t++) {
        const int r = min(16 * t + i16, m_rows - 1);
        lds_row[t] = r << units_shift;
        lds_mask[t] = r & kSwizzle;
    }

    f32x4 acc[MT][RT];
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
        for (int t = 0; t < RT; t++) acc[i][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    Fetched now, next;
    if (steps > 0) fetch(0, now);
    const int steps_per_stage = stage_cols / (128 * U * WK);
    for (int step = 0; step < steps; step++) {
        if (step % steps_per_stage == 0) {
            if (step) __syncthreads();
            stage(step * 128 * U * WK);
            __syncthreads();
        }
        if (step + 1 < steps) fetch(step + 1, next);
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int in_stage = (((step % steps_per_stage) * WK + wk) * U + u) * 128;
            uint32_t d[RT][4];
#pragma unroll
            for (int t = 0; t < RT; t++) {
#pragma unroll
                for (int j = 0; j < 4; j++) d[t][j] = now.w[u][t][j];
                // operand j of the whole wave has to lie within a group: a group of 128 takes word j of each lane as it comes
                if (GROUP < 128) transpose4(d[t]);
            }
#pragma unroll
            for (int g = 0; g < kGroups; g++) {
                Operand a[MT][kBlocks];
                Sum start[MT];
#pragma unroll
                for (int i = 0; i < MT; i++) {
                    start[i] = Sum{};
#pragma unroll
                    for (int j = 0; j < kBlocks; j++) {
                        const int unit = in_stage / 8 + (GROUP < 128 ? 4 * (g * kBlocks + j) + q : 4 * q + j);
                        a[i][j] = *reinterpret_cast<const Operand *>(lds + (lds_row[i] + (unit ^ lds_mask[i])) * kUnit);
                        if (A::kMoved) start[i] = A::product(a[i][j], A::minus24(), start[i]);
                    }
                }
#pragma unroll
                for (int t = 0; t < RT; t++) {
                    Operand b[kBlocks];
#pragma unroll
                    for (int j = 0; j < kBlocks; j++) b[j] = A::unfold(d[t][g * kBlocks + j]);
#pragma unroll
                    for (int i = 0; i < MT; i++) {
                        Sum s = start[i];
#pragma unroll
                        for (int j = 0; j < kBlocks; j++) s = A::product(a[i][j], b[j], s);
#pragma unroll
                        for (int r = 0; r < 4; r++) acc[i][t][r] = __builtin_fmaf((float)s[r], now.s[u][t][g], acc[i][t][r]);
                    }
                }
            }
        }
        now = next;
    }

    // join the waves that shared out the columns; element (m 4 q + r, row i16) of a tile is lane 16 q + i16's r-th
    __syncthreads();
    float *part = reinterpret_cast<float *>(lds);
    constexpr int kPerWave = MT * RT * 256;
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
        for (int t = 0; t < RT; t++)
            *reinterpret_cast<f32x4 *>(part + (wk * WN + wn) * kPerWave + ((i * RT + t) * 64 + lane) * 4) = acc[i][t];
    __syncthreads();
    for (int e = threadIdx.x; e < WN * kPerWave; e += kThreads) {
        // e: (wave of rows, tile, m within it, row within it), the row fastest
        const int w = e / kPerWave, tile = e % kPerWave / 256, mi = e % 256 / 16, ri = e % 16;
        const int mm = first_m + tile / RT * 16 + mi, row = (blockIdx.x * WN + w) * RT * 16 + tile % RT * 16 + ri;
        if (mm >= p.m || row >= p.rows) continue;
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < WK; k++) v += part[(k * WN + w) * kPerWave + (tile * 64 + mi / 4 * 16 + ri) * 4 + mi % 4];
        if (p.x_scales) v *= A::kUnit * p.x_scales[mm];
        const int64_t at = (int64_t)mm * p.rows + row;
        if (p.y_dtype == GQ_F32) ((float *)p.y)[at] = p.bias ? v + ((const float *)p.bias)[row] : v;
        else if (p.y_dtype == GQ_BF16) ((bf16 *)p.y)[at] = (bf16)(p.bias ? v + (float)((const bf16 *)p.bias)[row] : v);
        else ((f16 *)p.y)[at] = (f16)(p.bias ? v + (float)((const f16 *)p.bias)[row] : v);
    }
}

template <typename X, typename S, int GROUP, int MT, int RT, int WN, int WK, int U>
static gq_status launch_matvec(MatvecArgs p, hipStream_t stream)
{
    constexpr int kStep = 128 * U * WK, kLimit = 64 * 1024;
    const int m_rows = p.m < MT * 16 ? p.m : MT * 16;
    static_assert(MT * 16 * kStep * (int)sizeof(X) <= kLimit && WN * WK * MT * RT * 1024 <= kLimit, "LDS");
    p.stage_shift = __builtin_ctz(kStep);
    while ((1 << p.stage_shift) < p.cols && (m_rows << (p.stage_shift + 1)) * (int)sizeof(X) <= kLimit) p.stage_shift++;
    const unsigned staged = (unsigned)(m_rows << p.stage_shift) * (unsigned)sizeof(X), joined = WN * WK * MT * RT * 1024;
    const int64_t bx = ((int64_t)p.rows + WN * RT * 16 - 1) / (WN * RT * 16), by = ((int64_t)p.m + MT * 16 - 1) / (MT * 16);
    if (!grid_fits(bx, 64 * WN * WK) || by > 65535) return GQ_ERR_INVALID_ARG;
    w4_matvec_kernel<X, S, GROUP, MT, RT, WN, WK, U><<<dim3((unsigned)bx, (unsigned)by), 64 * WN * WK, staged > joined ? staged : joined, stream>>>(p);
    return launched();
}

template <typename X, typename S, int GROUP> static gq_status matvec_by_rows(const MatvecArgs &p, hipStream_t stream)
{
    if (p.m <= 16) return launch_matvec<X, S, GROUP, 1, 1, 1, 8, 2>(p, stream);
    if (p.m <= 32) return launch_matvec<X, S, GROUP, 2, 2, 2, 4, 2>(p, stream);
    return launch_matvec<X, S, GROUP, 4, 2, 2, 4, 1>(p, stream);
}

}  // namespace gq

using namespace gq;

extern "C" gq_status gq_w4_matvec(const void *x, const float *x_scales, int64_t m, gq_dtype x_dtype, const void *codes, const void *scales,
                                  gq_dtype scale_dtype, int64_t rows, int64_t cols, int group, const void *bias, void *y, gq_dtype y_dtype,
                                  void *hip_stream)
{
    const gq_status st = check_weights(rows, cols, group, scale_dtype);
    if (st != GQ_OK) return st;
    if ((x_dtype != GQ_BF16 && x_dtype != GQ_F16 && x_dtype != GQ_I8) || !float_type(y_dtype) || (x_dtype == GQ_I8) != (x_scales != nullptr) ||
        !matrix_fits(m, cols) || !matrix_fits(m, rows)) return GQ_ERR_INVALID_ARG;
    if (m == 0 || rows == 0) return GQ_OK;
    if (!aligned(y, 16) || !aligned_or_null(bias, 16) || (cols > 0 && (!aligned(x, 16) || !aligned(codes, 16) || !aligned(scales, 16))) ||
        !aligned_or_null(x_scales, 4)) return GQ_ERR_INVALID_ARG;
    const MatvecArgs p = {x, x_scales, (const uint8_t *)codes, scales, bias, y, gq_w4_row_bytes(cols), (int)m, (int)rows, (int)cols,
                          (int)((cols + group - 1) / group), (int)y_dtype, 0};
    const hipStream_t stream = (hipStream_t)hip_stream;
    return with_scale_type(scale_dtype, [&](auto s) {
        typedef decltype(s) S;
        auto go = [&](auto t) {
            typedef decltype(t) X;
            return group == 32 ? matvec_by_rows<X, S, 32>(p, stream) : group == 64 ? matvec_by_rows<X, S, 64>(p, stream) : matvec_by_rows<X, S, 128>(p, stream);
        };
        return x_dtype == GQ_BF16 ? go(bf16()) : x_dtype == GQ_F16 ? go(f16()) : go(int8_t());
    });
}
