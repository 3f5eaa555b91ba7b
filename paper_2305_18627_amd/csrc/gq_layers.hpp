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
// Kept as words: an element a register is what becomes of them otherwise where a guarded and an unguarded load meet.
template <typename T> struct Eight {
    uint32_t w __attribute__((ext_vector_type(2 * sizeof(T))));
    __device__ __forceinline__ float f(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        const uint32_t v = w[i / 2];
        if constexpr (std::is_same<T, bf16>::value) return __uint_as_float((i & 1) ? v & 0xFFFF0000u : v << 16);
        return (float)__builtin_bit_cast(f16, (uint16_t)((i & 1) ? v >> 16 : v));
    }
};
// 16 bytes at an address that is a multiple of an element's size
template <size_t SIZE> struct Chunk;
template <> struct Chunk<4> { typedef uint32_t bits; typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Chunk<2> { typedef uint16_t bits; typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2))); };

// t without its first `over` elements, zeros behind: by 4, 2 and 1 of them
template <int WORDS, typename T> __device__ __forceinline__ void drop_words(Eight<T> &t, bool really)
{
    constexpr int kWords = 2 * sizeof(T);
#pragma unroll
    for (int i = 0; i < kWords; i++) {
        const uint32_t from = i + WORDS < kWords ? t.w[(i + WORDS) % kWords] : 0u;
        t.w[i] = really ? from : t.w[i];
    }
}
template <typename T> __device__ __forceinline__ void drop_low(Eight<T> &t, int64_t over)
{
    constexpr int kWords = 2 * sizeof(T), kPer = 4 / sizeof(T);
    drop_words<4 / kPer>(t, over & 4);
    drop_words<2 / kPer>(t, over & 2);
    if constexpr (kPer == 1) {
        drop_words<1>(t, over & 1);
    } else {
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            const uint32_t from = (t.w[i] >> 16) | (i + 1 < kWords ? t.w[(i + 1) % kWords] << 16 : 0u);
            t.w[i] = (over & 1) ? from : t.w[i];
        }
    }
#pragma unroll
    for (int i = 0; i < kWords; i++) t.w[i] = over < 8 ? t.w[i] : 0u;
}

// Columns c .. c + 7 of a row of n.  ask8() loads without a branch per lane: a unit that runs over the row's end (or lies past it) is
// read so that it ends there, and settle8() moves it into place, zeros past the end.  Between the two the caller asks for more: a
// load behind a branch would be waited for there.  ONCE: what no other row reads again; non-temporal,
// but for binary32, of which an instruction takes every other 16 bytes: 8192x4096 norm 105 -> 98 us, 8192x8192 dropout 104 -> 96 without.
// TINY: rows of fewer than eight columns; they have kernels of their own, for this way through, with its branches and waits, slows the
// other one down even where it is not taken.
template <bool ONCE, bool TINY, typename T> __device__ __forceinline__ void ask8(const T *row, int64_t n, int64_t c, Eight<T> &t)
{
    typedef typename Chunk<sizeof(T)>::type V;
    typedef typename Chunk<sizeof(T)>::bits Bits;
    constexpr int kWords = 2 * sizeof(T), kPer = 4 / sizeof(T);
    if (!TINY) {
        const V *at = reinterpret_cast<const V *>(row + (c < n - 8 ? c : n - 8));
#pragma unroll
        for (int i = 0; i < kWords / 4; i++) {
            const V v = ONCE && sizeof(T) == 2 ? __builtin_nontemporal_load(at + i) : at[i];
#pragma unroll
            for (int j = 0; j < 4; j++) t.w[4 * i + j] = v[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < kWords; j++) {
            t.w[j] = 0u;
#pragma unroll
            for (int i = 0; i < kPer; i++)
                if (c + kPer * j + i < n) t.w[j] |= (uint32_t) reinterpret_cast<const Bits *>(row)[c + kPer * j + i] << (8 * sizeof(T) * i);
        }
    }
}
template <bool TINY, typename T> __device__ __forceinline__ void settle8(int64_t n, int64_t c, Eight<T> &t)
{
    if (!TINY && c > n - 8) drop_low(t, c - (n - 8));
}
template <typename T> __device__ __forceinline__ void store8(T *p, int64_t left, const float *v)
{
    typedef typename Chunk<sizeof(T)>::type V;
    struct { T e[8]; } t;
#pragma unroll
    for (int i = 0; i < 8; i++) t.e[i] = (T)v[i];                      // to nearest even
    if (left >= 8) {
#pragma unroll
        for (size_t i = 0; i < sizeof(t) / 16; i++) {
            V c;
            __builtin_memcpy(&c, reinterpret_cast<const char *>(&t) + 16 * i, 16);
            if (sizeof(T) == 2) __builtin_nontemporal_store(c, reinterpret_cast<V *>(p) + i);
            else reinterpret_cast<V *>(p)[i] = c;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < left) p[i] = t.e[i];
    }
}

// Row and unit within it of a lane's k-th unit, where rows have `per_row` units and a workgroup takes UNITS * kBlock of them: one
// 64-bit division a workgroup, on the scalar unit, and a 32-bit one a unit.  FLAT: all is one row of less than 2^31 units (whole units a
// row make a matrix one), nothing is divided.  The row may lie past the last one.
struct RowUnit { int64_t row; uint32_t unit; };
template <int UNITS, bool FLAT> __device__ __forceinline__ RowUnit row_unit(uint32_t block, int k, uint32_t per_row)
{
    if constexpr (FLAT) {
        const uint32_t u = block * (UNITS * kBlock) + (uint32_t)k * kBlock + threadIdx.x;
        return {u >= per_row, u};
    }
    const uint64_t first = (uint64_t)block * (UNITS * kBlock), row = first / per_row;
    const uint32_t at = (uint32_t)(first - row * per_row) + (uint32_t)k * kBlock + threadIdx.x;    // below 2^28 + 2^12 for a matrix that fits
    const uint32_t more = at / per_row;
    return {(int64_t)row + more, at - more * per_row};
}
// f(first row, rows) for as many rows at a time as one launch covers, `units` units a lane: all of them but for 2^32 units and more
template <typename F> static inline gq_status in_launches(int64_t rows, int64_t per_row, int units, F &&f)
{
    const int64_t most = (0xFFFFFFFFLL / kBlock * kBlock) * units / per_row;
    for (int64_t first = 0; first < rows; first += most) {
        const gq_status st = f(first, rows - first < most ? rows - first : most);
        if (st != GQ_OK) return st;
    }
    return GQ_OK;
}
static inline bool flat_fits(int64_t units) { return units < 0x7FFFFFFF - 4096; }

// The dropout decision of gq_dropout_params, as the kernels take it.
struct Drop {
    uint32_t k0, k1, worker;
    uint32_t threshold;   // dropped iff the draw (32 bits, or 16 moved to the top of 32) is below it
    uint64_t first;       // index_base
    float scale;          // of what is kept
};

// the draws of the elements g .. g + 7 of the stream (g a multiple of 4, of 8 with short draws)
template <bool SHORT> __device__ __forceinline__ void draws8(const Drop &d, uint64_t g, uint32_t *r)
{
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
}
__device__ __forceinline__ float dropped(const Drop &d, uint32_t draw, float v) { return draw >= d.threshold ? v * d.scale : 0.0f; }
// v[0..7], the elements g .. g + 7, after dropout
template <bool SHORT> __device__ __forceinline__ void drop8(const Drop &d, uint64_t g, float *v)
{
    uint32_t r[8];
    draws8<SHORT>(d, g, r);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = dropped(d, r[i], v[i]);
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
constexpr int64_t kMaxWeightCols = 1 << 24;
static inline gq_status check_weights(int64_t rows, int64_t cols, int group, int scale_dtype)
{
    if (!matrix_fits(rows, cols) || rows > (1 << 30) || cols > kMaxWeightCols || (group != 32 && group != 64 && group != 128)) return GQ_ERR_INVALID_ARG;
    return scale_dtype == GQ_F32 || scale_dtype == GQ_BF16 ? GQ_OK : GQ_ERR_INVALID_ARG;
}
template <typename F> static inline gq_status with_scale_type(int t, F &&f) { return t == GQ_F32 ? f(float()) : f(bf16()); }

}  // namespace gq
