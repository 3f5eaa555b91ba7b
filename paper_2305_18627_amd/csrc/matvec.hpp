// Rows of activations times 4-bit weights under group scales, on the matrix cores: the kernel and the choice of its shape, compiled
// once for each type of activations (matvec_bf16.hip, matvec_f16.hip, matvec_i8.hip).
// The contract of the entry point is stated in include/gqsgd.h.
#pragma once
#include "gq_layers.hpp"

namespace gq {

// What an activation type brings along.  A lane's eight codes are one word; the instructions take them as eight activations'
// worth of operand B, and x as operand A in the order in which unfolding leaves the codes:
//   16 bits  pairs (i, i + 4): a shift brings nibbles i and i + 4 of the word behind the exponent of 16.0 of two halves, one three-input
//            instruction masks them, flips their top bits (two's complement becomes code + 8) and sets the exponent: the halves are
//            then 16 + (code + 8) = 24 + code exactly.  24 times the sum of x is taken out again by the same products with a constant
//            operand of -24.
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
    // the two constants in a scalar and a vector register, as one instruction can take them
    struct Constants {
        uint32_t mask, flip;
        __device__ __forceinline__ Constants() : mask(0x000F000Fu << TOP), flip(ONE ^ (0x00080008u << TOP))
        {
            asm volatile("" : "+s"(mask));
            asm volatile("" : "+v"(flip));
        }
    };
    static __device__ __forceinline__ Operand unfold(uint32_t w, const Constants &c)
    {
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int by = 4 * i - TOP;                                // to the right
            const uint32_t t = by >= 0 ? w >> (by & 31) : w << (-by & 31);
            r[i] = __builtin_amdgcn_bitop3_b32(t, c.mask, c.flip, 0x6A);   // (t & mask) ^ flip
        }
        return __builtin_bit_cast(Operand, r);
    }
    static __device__ __forceinline__ Operand minus24() { return __builtin_bit_cast(Operand, u32x4{MINUS, MINUS, MINUS, MINUS}); }
    // eight activations as they lie in memory, and in the order of unfold()
    typedef u32x4 Raw;
    typedef uint16_t Bits;
    static __device__ __forceinline__ Raw ordered(Raw v)
    {
        return Raw{(v.x & 0xFFFFu) | (v.z << 16), (v.x >> 16) | (v.z & 0xFFFF0000u), (v.y & 0xFFFFu) | (v.w << 16), (v.y >> 16) | (v.w & 0xFFFF0000u)};
    }
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
    struct Constants {};
    static __device__ __forceinline__ Operand unfold(uint32_t w, const Constants &)
    {
        return __builtin_bit_cast(Operand, u32x2{(w << 4) & 0xF0F0F0F0u, w & 0xF0F0F0F0u});
    }
    static __device__ __forceinline__ Sum product(Operand a, Operand b, Sum c) { return __builtin_amdgcn_mfma_i32_16x16x32_i8(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ Operand minus24() { return 0; }
    typedef u32x2 Raw;
    typedef uint8_t Bits;
    static __device__ __forceinline__ Raw ordered(Raw v)
    {
        return Raw{__builtin_amdgcn_perm(v.y, v.x, 0x06040200u), __builtin_amdgcn_perm(v.y, v.x, 0x07050301u)};
    }
};

__device__ __forceinline__ bool is_finite(float f) { return __builtin_fabsf(f) <= 3.402823466e+38f; }

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
    int m, rows, cols, groups, y_dtype;
    int row_shift;        // a row of staged x in LDS has 2^row_shift columns
};

// y = x times the transposed weights: 2 m rows cols operations on rows cols / 2 bytes of codes, which are read once for all rows of x of a
// slice.  Bound by these bytes for a row or a few (28672x8192, int8, 132 MB with scales: 27.9 us, 4.7 TB/s; a bare read of such codes
// takes 22); for more rows by what a step costs beside them and does not overlap (61 rows, 14335x4095, fp16, groups of 32: 28.9 us, 248
// TFLOP/s: vector instructions take 54 % of the cycles, matrix instructions 27 %, LDS 25 %); for small matrices by latency (4096x4096: 4.7
// us).  These are kernels of a captured graph, one after another; calls from a program overlap at their ends and take up to 3 us less.
// A workgroup of WN x WK waves owns WN * 16 rows of the weights at a time and up to MT * 16 rows of x; the WK waves share out
// the columns, 128 U at a time (a step), and their sums are joined in LDS at a tile's end.  x is staged in LDS: RESIDENT, all of
// it, once, for all tiles of rows that the workgroup takes in turn; otherwise a step's columns at a time into two buffers in
// turn, the next step's loads in flight meanwhile, and the workgroup takes one tile.
template <typename X, typename S, int GROUP, int MT, int WN, int WK, int U, bool RESIDENT>
__global__ void __launch_bounds__(64 * WN * WK)
w4_matvec_kernel(MatvecArgs p)
{
    typedef Act<X> A;
    typedef typename A::Operand Operand;
    typedef typename A::Sum Sum;
    typedef typename A::Raw Raw;
    typedef typename A::Bits Bits;
    constexpr int kThreads = 64 * WN * WK, kUnit = 8 * (int)sizeof(X), kSwizzle = 128 / kUnit - 1;
    constexpr int kGroups = 128 / GROUP, kBlocks = GROUP / 32, kStep = 128 * U * WK;
    constexpr int kPerWave = MT * 256, kPart = WN * WK * kPerWave;            // floats of the waves' sums
    constexpr int kBuffer = MT * 16 * kStep * (int)sizeof(X);
    constexpr int kAhead = MT * 16 * (kStep / 8) / kThreads;                       // units of a step's x per lane
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    // the wave's number on the scalar unit, and with it all addresses that its lanes share
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = wave % WK, wn = wave / WK;
    const typename A::Constants constants;
    const int i16 = lane & 15, q = lane >> 4;
    const int first_m = blockIdx.y * MT * 16, m_rows = min(p.m - first_m, MT * 16);
    const X *x = (const X *)p.x + (int64_t)first_m * p.cols;
    const int tiles = (p.rows + WN * 16 - 1) / (WN * 16), steps = (p.cols + kStep - 1) / kStep;

    // ---- x: units of eight columns, in the order in which the codes unfold ----
    auto load_unit = [&](int row, int c) {
        Raw v;
        const X *at = x + (int64_t)row * p.cols + c;
        if (c + 8 <= p.cols) {
            __builtin_memcpy(&v, at, sizeof(v));
        } else {
            constexpr int kBits = 8 * (int)sizeof(X), kWord = 32 / kBits;
            v = Raw{};
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (c + i < p.cols) v[i / kWord] |= (uint32_t) reinterpret_cast<const Bits *>(at)[i] << (kBits * (i % kWord));
        }
        return v;
    };
    // v without its first `over` elements, zeros behind; v itself for over <= 0
    auto drop_low = [&](Raw v, int over) {
        if (over <= 0) return v;
        constexpr int kWords = sizeof(Raw) / 4, kBits = 8 * (int)sizeof(X);
        const int bits = min(over, 8) * kBits, words = bits / 32, rest = bits % 32;
        uint32_t w[2 * kWords + 1];
#pragma unroll
        for (int i = 0; i <= 2 * kWords; i++) w[i] = i < kWords ? v[i] : 0u;
        Raw o;
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            uint32_t lo = 0, hi = 0;
#pragma unroll
            for (int k = 0; k <= kWords; k++) {
                lo = words == k ? w[i + k] : lo;
                hi = words == k ? w[i + k + 1] : hi;
            }
            o[i] = (uint32_t)((((uint64_t)hi << 32) | lo) >> rest);
        }
        return o;
    };
    auto store_unit = [&](uint8_t *to, int row, int unit, int shift, Raw v) {
        *reinterpret_cast<Raw *>(to + ((row << shift) + (unit ^ (row & kSwizzle))) * kUnit) = A::ordered(v);
    };
    const int shift = RESIDENT ? p.row_shift - 3 : __builtin_ctz(kStep / 8);       // of units a row
    // where a lane finds operand A: unit 16 chunk + (4 j + q), or (4 q + j) for groups of 128, of its row; a chunk is 128 columns.
    // Rows of x that are not there are the last one again and end in rows of y that are not there.
    int from[4];
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const int r = RESIDENT ? min(i16, m_rows - 1) : i16;
        from[j] = ((r << shift) + ((GROUP < 128 ? 4 * j + q : 4 * q + j) ^ (r & kSwizzle))) * kUnit;
    }
    constexpr int kTileBytes = 16 * kStep * (int)sizeof(X);                        // of 16 rows of x, streamed

    // ---- codes and scales of a step: 16 bytes of codes a lane and chunk, the scales of its row's chunks in one load ----
    // Both stay as they lie in memory until they are used: a conversion here would be waited for here.
    constexpr int kScales = U * kGroups, kScaleWords = (kScales * (int)sizeof(S) + 3) / 4;
    struct Fetched { u32x4 w[U]; uint32_t s[kScaleWords]; };
    const uint32_t scale_bytes = (uint32_t)(p.groups * (int)sizeof(S));
    const int last_block = (p.cols - 1) / 32;
    // the first scale of a step's load: where the step runs over the row's end, so early that the load does not
    auto first_scale = [&](int step) { return min((step * WK + wk) * kScales, max(p.groups - kScales, 0)); };
    auto fetch = [&](int tile, int step, Fetched &f) {
        // The wave's first row is the same for all lanes, what differs is a lane's row within the tile.  A wave whose rows all lie past
        // the last one reads that one, and so do rows past it: never stored.
        const int first = min((tile * WN + wn) * 16, p.rows - 1), c = (step * WK + wk) * U * 128;
        const uint8_t *codes = p.codes + (int64_t)first * p.row_bytes;
        const uint8_t *scales = (const uint8_t *)p.scales + ((int64_t)first * p.groups + first_scale(step)) * (int)sizeof(S);
        const int last = p.rows - 1 - first;
        const uint32_t r = (uint32_t)min(i16, last), at = r * (uint32_t)p.row_bytes;
        // past the row's end the last codes again, where x is zero
#pragma unroll
        for (int u = 0; u < U; u++)
            f.w[u] = *reinterpret_cast<const u32x4 *>(codes + (at + 16u * (uint32_t)min(c / 32 + 4 * u + q, last_block)));
        if (p.groups >= kScales) {
            if constexpr (kScaleWords * 4 != kScales * (int)sizeof(S)) f.s[kScaleWords - 1] = 0;
            __builtin_memcpy(f.s, scales + r * scale_bytes, kScales * sizeof(S));
        } else {                                                                   // few columns
            typedef typename std::conditional<sizeof(S) == 4, uint32_t, uint16_t>::type Bits;
            constexpr int kPer = 4 / (int)sizeof(S);
            const Bits *from_row = reinterpret_cast<const Bits *>(scales + r * scale_bytes);
#pragma unroll
            for (int j = 0; j < kScaleWords; j++) {
                f.s[j] = 0;
#pragma unroll
                for (int i = 0; i < kPer; i++)
                    if (j * kPer + i < p.groups) f.s[j] |= (uint32_t)from_row[j * kPer + i] << (16 * i);
            }
        }
    };
    // a step's scales as numbers, zeros behind the row's end
    auto scales_of = [&](const uint32_t *words, int step, float *s) {
#pragma unroll
        for (int k = 0; k < kScales; k++) {
            if constexpr (sizeof(S) == 4) s[k] = __uint_as_float(words[k]);
            else s[k] = __uint_as_float((k & 1) ? words[k / 2] & 0xFFFF0000u : words[k / 2] << 16);
        }
        // what the load began too early, or what lies behind the row's end where it could not begin earlier
        for (int late = min((step * WK + wk) * kScales - first_scale(step), kScales); late > 0; late--) {
#pragma unroll
            for (int k = 0; k < kScales; k++) s[k] = k + 1 < kScales ? s[k + 1] : 0.0f;
        }
    };

    f32x4 acc[MT];
    auto clear = [&] {
#pragma unroll
        for (int i = 0; i < MT; i++) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    };
    // a step's products; `staged`: where its first column is
    auto multiply = [&](const Fetched &f, int step, const uint8_t *staged) {
        float scale[kScales];
        scales_of(f.s, step, scale);
#pragma unroll
        for (int u = 0; u < U; u++) {
            const uint8_t *chunk = staged + (wk * U + u) * 16 * kUnit;
            uint32_t d[4] = {f.w[u].x, f.w[u].y, f.w[u].z, f.w[u].w};
            // operand j of the whole wave has to lie within a group: a group of 128 takes word j of each lane as it comes
            if (GROUP < 128) transpose4(d);
#pragma unroll
            for (int g = 0; g < kGroups; g++) {
                Sum sum[MT];
#pragma unroll
                for (int i = 0; i < MT; i++) sum[i] = Sum{};
#pragma unroll
                for (int j = g * kBlocks; j < (g + 1) * kBlocks; j++) {
                    const Operand b = A::unfold(d[j], constants);
#pragma unroll
                    for (int i = 0; i < MT; i++) {
                        const Operand a = *reinterpret_cast<const Operand *>(chunk + from[j] + i * kTileBytes);
                        if (A::kMoved) sum[i] = A::product(a, A::minus24(), sum[i]);
                        sum[i] = A::product(a, b, sum[i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < MT; i++)
#pragma unroll
                    for (int r = 0; r < 4; r++) acc[i][r] = __builtin_fmaf((float)sum[i][r], scale[u * kGroups + g], acc[i][r]);
                // the groups one after another, sums and all: left to itself the compiler moves all sums behind all products, and
                // the products of all groups at once are more than the registers that there are
                if (MT > 1) {
#pragma unroll
                    for (int i = 0; i < MT; i++) asm volatile("" : "+v"(acc[i]));
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    };
    // the waves that shared out the columns leave their sums in `part`; element (m 4 q + r, row i16) of a tile is lane 16 q + i16's r-th
    auto leave = [&](float *part) {
#pragma unroll
        for (int i = 0; i < MT; i++) *reinterpret_cast<f32x4 *>(part + (wk * WN + wn) * kPerWave + (i * 64 + lane) * 4) = acc[i];
    };
    // Products whose sums are not finite, once more in binary64: the sums of 24 |x| of a bfloat16 row, and 16 times the sum of int8 codes, may
    // leave binary32 where the product does not.  One after another, the whole wave at each; a row of x that is not finite ends it for all its
    // products, a scale of NaN, looked for first, for this one.  A column a lane, in few registers, for it is rare: 64 rows of x,
    // 28672x8192, groups of 64, take 20 ms where all products go this way, 1.3 where each row of x ends in an infinity, 0.08 otherwise.
    auto once_more = [&](bool wanted, int row_of_x, int row, float &v) {
        for (uint64_t left = __ballot(wanted && !is_finite(v)); left != 0;) {
            const int l = __builtin_ctzll(left), rx = __builtin_amdgcn_readlane(row_of_x, l), rw = __builtin_amdgcn_readlane(row, l);
            const X *at = x + (int64_t)rx * p.cols;
            const uint8_t *codes = p.codes + rw * p.row_bytes;
            const S *scales = (const S *)p.scales + (int64_t)rw * p.groups;
            double s = 0.0;
            bool finite = true;
#pragma unroll 1
            for (int g = lane; g < p.groups; g += 64)
                if (const float scale = (float)scales[g]; scale != scale) s = __builtin_nan("");
#pragma unroll 1
            for (int first = 0; first < p.cols && __all(finite && s == s); first += 64) {
                const uint32_t c = (uint32_t)min(first + lane, p.cols - 1);
                const float f = first + lane < p.cols ? (float)at[c] : 0.0f;
                finite = is_finite(f);
                s += (double)f * ((double)(float)scales[c / GROUP] * (double)((int)((uint32_t)codes[c / 2] << (28 - 4 * (c & 1))) >> 28));
            }
            const bool nan = !__all(finite);
            s = wave_sum(s);
            if (nan ? row_of_x == rx : lane == l) v = nan ? __builtin_nanf("") : (float)s;
            left &= nan ? ~__ballot(row_of_x == rx) : left - 1;
        }
    };
    auto join = [&](const float *part, int tile_of_rows) {
        for (int e = threadIdx.x; e < WN * kPerWave; e += kThreads) {
            // e: (wave of rows, tile, m within it, row within it), the row fastest
            const int w = e / kPerWave, tile = e % kPerWave / 256, mi = e % 256 / 16, ri = e % 16;
            const int mm = first_m + tile * 16 + mi, row = (tile_of_rows * WN + w) * 16 + ri;
            const bool there = mm < p.m && row < p.rows;
            float v = 0.0f;
#pragma unroll
            for (int k = 0; k < WK; k++) v += part[(k * WN + w) * kPerWave + (tile * 64 + mi / 4 * 16 + ri) * 4 + mi % 4];
            if (!A::kMoved) v *= A::kUnit;
            if constexpr (!std::is_same<X, f16>::value) once_more(there, mm - first_m, row, v);      // binary16 is too small for either
            if (!there) continue;
            // the 16 of int8 sums has been taken out of the sum: the row's scale may be subnormal, and its product with 1 / 16 is then rounded
            if (p.x_scales) v *= p.x_scales[mm];
            const int64_t at = (int64_t)mm * p.rows + row;
            if (p.y_dtype == GQ_F32) ((float *)p.y)[at] = p.bias ? v + ((const float *)p.bias)[row] : v;
            else if (p.y_dtype == GQ_BF16) ((bf16 *)p.y)[at] = (bf16)(p.bias ? v + (float)((const bf16 *)p.bias)[row] : v);
            else ((f16 *)p.y)[at] = (f16)(p.bias ? v + (float)((const f16 *)p.bias)[row] : v);
        }
    };

    if constexpr (RESIDENT) {
        Fetched now, next;
        // the first units of x are asked for before the codes: loads come back in order, and x is wanted first
        const int units = m_rows << shift;
        constexpr int kFirst = 2;
        Raw v[kFirst];
#pragma unroll
        for (int i = 0; i < kFirst; i++) {
            const int u = min((int)threadIdx.x + i * kThreads, units - 1);
            v[i] = load_unit(u >> shift, (u & ((1 << shift) - 1)) * 8);
        }
        if (steps > 0) fetch(blockIdx.x, 0, now);
#pragma unroll
        for (int i = 0; i < kFirst; i++) {
            const int u = (int)threadIdx.x + i * kThreads;
            if (u < units) store_unit(lds, u >> shift, u & ((1 << shift) - 1), shift, v[i]);
        }
        for (int u = threadIdx.x + kFirst * kThreads; u < units; u += kThreads)
            store_unit(lds, u >> shift, u & ((1 << shift) - 1), shift, load_unit(u >> shift, (u & ((1 << shift) - 1)) * 8));
        __syncthreads();
        float *parts = reinterpret_cast<float *>(lds + units * kUnit);             // two, in turn
        int turn = 0;
        for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x, turn ^= 1) {
            clear();
            for (int step = 0; step < steps; step++) {
                const bool more = step + 1 < steps;
                if (more || tile + (int)gridDim.x < tiles) fetch(more ? tile : tile + gridDim.x, more ? step + 1 : 0, next);
                multiply(now, step, lds + step * (kStep / 8) * kUnit);
                now = next;
            }
            // one barrier a tile: who writes a part again has passed the next tile's, and so have all who read it
            leave(parts + turn * kPart);
            __syncthreads();
            join(parts + turn * kPart, tile);
        }
    } else {
        // a lane's units are in one column of units, kRowsApart rows apart; rows that are not there hold the last one again
        constexpr int kRowUnits = kStep / 8, kRowsApart = kThreads / kRowUnits;
        static_assert(kThreads % kRowUnits == 0 && kAhead * kRowsApart == MT * 16, "units of a step");
        const int unit = threadIdx.x % kRowUnits, row0 = threadIdx.x / kRowUnits;
        Raw ahead[kAhead];
        // rows of fewer than eight columns are read in put(); what is asked for here is then 16 bytes of codes, not used
        const X *asked = p.cols < 8 ? (const X *)p.codes : x;
        const int apart = p.cols < 8 ? 0 : p.cols;
        // a unit that runs over the row's end (or lies past it) is read so that it ends there, and moved into place in put()
        auto ask = [&](int step) {
            const int c = p.cols < 8 ? 0 : min(step * kStep + 8 * unit, p.cols - 8);
#pragma unroll
            for (int i = 0; i < kAhead; i++)
                __builtin_memcpy(&ahead[i], asked + (uint32_t)(min(row0 + i * kRowsApart, m_rows - 1) * apart + c), sizeof(Raw));
        };
        auto put = [&](int step) {
            uint8_t *to = lds + (step & 1) * kBuffer;
            if (p.cols < 8) {
                for (int i = 0; i < kAhead; i++)
                    store_unit(to, row0 + i * kRowsApart, unit, shift, load_unit(min(row0 + i * kRowsApart, m_rows - 1), 8 * unit));
                return;
            }
            if ((step + 1) * kStep > p.cols) {
                const int over = step * kStep + 8 * unit - (p.cols - 8);           // elements to drop from the low end
#pragma unroll
                for (int i = 0; i < kAhead; i++) ahead[i] = drop_low(ahead[i], over);
            }
#pragma unroll
            for (int i = 0; i < kAhead; i++) store_unit(to, row0 + i * kRowsApart, unit, shift, ahead[i]);
        };
        // Codes are asked for two steps ahead, x one.  No branch is around a load, for what is loaded on one way only is waited for where the
        // ways join: past the last step its loads come again.  us before and after, as measured when this was added: 61 rows of x, 14335x4095, groups of 32,
        // f16 34.3 and 29.8; 64 rows, 8192x8192 29.7, 26.9; 64x14000 33.7, 28.3.  Three sets of codes only as far as 128
        // registers reach (else they spill: 32 rows, 4096x4096, groups of 32 9.0 and 13.4): 45 words of codes, scales and x, or 56 where the
        // groups' products stay apart and a lane's x is little; and not for 16 rows in int8 (12.6, 13.7).
        constexpr int kWords = 3 * (4 * U + kScaleWords) + kAhead * (int)sizeof(Raw) / 4;
        constexpr int kSets = MT <= 2 && sizeof(X) * MT >= 2 && kWords <= (MT == 2 && WK == 2 ? 56 : 45) ? 3 : 2;
        Fetched f[kSets];
        clear();
        if (steps > 0) {
            ask(0);
#pragma unroll
            for (int k = 0; k + 1 < kSets; k++) fetch(blockIdx.x, min(k, steps - 1), f[k]);
            put(0);
        }
        __syncthreads();
        for (int step = 0; step < steps;) {
#pragma unroll
            for (int k = 0; k < kSets; k++) {
                ask(min(step + 1, steps - 1));
                fetch(blockIdx.x, min(step + kSets - 1, steps - 1), f[(k + kSets - 1) % kSets]);
                multiply(f[k], step, lds + (step & 1) * kBuffer);
                if (step + 1 < steps) put(step + 1);         // last read two steps ago, before the barrier that ended that step
                __syncthreads();
                if (++step >= steps) break;
            }
        }
        float *part = reinterpret_cast<float *>(lds);
        leave(part);
        __syncthreads();
        join(part, blockIdx.x);
    }
}

template <typename X, typename S, int GROUP, int MT, int WN, int WK, int U, bool RESIDENT>
static gq_status launch_matvec(const MatvecArgs &p, hipStream_t stream)
{
    constexpr int kStep = 128 * U * WK, kParts = WN * WK * MT * 1024, kRows = WN * 16;
    const int resident_groups = p.m <= 2 ? 768 : 512;                              // two or three a compute unit: each takes its tiles in turn
    static_assert(2 * MT * 16 * kStep * (int)sizeof(X) <= 128 * 1024 && kParts <= 128 * 1024, "LDS");
    int64_t bx = ((int64_t)p.rows + kRows - 1) / kRows;
    const int64_t by = ((int64_t)p.m + MT * 16 - 1) / (MT * 16);
    unsigned lds;
    if (RESIDENT) {
        lds = (unsigned)((p.m << p.row_shift) * (int)sizeof(X) + 2 * kParts);
        if (bx > resident_groups) bx = resident_groups;
    } else {
        lds = 2 * MT * 16 * kStep * (int)sizeof(X);
        if (lds < kParts) lds = kParts;
    }
    if (!grid_fits(bx, 64 * WN * WK)) return GQ_ERR_INVALID_ARG;
    w4_matvec_kernel<X, S, GROUP, MT, WN, WK, U, RESIDENT><<<dim3((unsigned)bx, (unsigned)by), 64 * WN * WK, lds, stream>>>(p);
    return launched();
}

// Which shape of workgroup.  Few rows of x stay in LDS.  us, bf16, groups of 128; WK waves that take U chunks each:
//   1 row of x    4096x4096  16 waves of 1 chunk 4.8, 8 of 2 5.3, 4 of 4 5.3  (too few tiles for more than one workgroup a compute unit)
//                14336x4096  4 of 4 9.4, 8 of 2 9.7, 16 of 1 12.7;  2 rows of x: 10.8, 9.6, 13.6;  4: 12.5, 11.0, 11.7
//                28672x8192  8 of 2 25.9, 4 of 4 28.3, 16 of 1 32.7
//   8 rows of x, 14336x4096: 512 workgroups 13.4, 768: 18
// Otherwise as many rows of weights a workgroup (they share its staged x) as leave no more than one workgroup a compute unit, 256 in all, and as
// many waves to share out the columns as fill it: one workgroup more starts a second round.  us, 16 | 32 | 64 rows of x, by the rows of
// weights a workgroup (and the rows of x in its slice, where that is less):
//   4096x4096    16: 6.6, 32: 9.2, 64: 12.1   |  32 (16) 9.6, 16 (16) 11.4, 32 12.3        |  32 (32) 12.7, 64 (32) 14.4, 32 (16) 17.7
//   5120x4096    32: 9.3, 16: 11.1, 64: 12.2  |  32: 12.4, 64 14.3, 32 (16) 16.9           |  64 (32) 14.2, 128 (32) 20.1, 32 (32) 22.1
//   8192x8192    32: 17.2, 64: 21.8, 16: 22.6 |  32: 23.3, 64 (16) 22.2, 64 26.0           |  64 (32) 26.5, 128 (32) 40.0, 32 (32) 42.3
//   10240x4096   64: 13.1, 32: 17.7, 16: 18.5 |  64: 15.4, 128 21.9, 32 24.7               |  128 (32) 22.1, 64 (32) 27.9, 128 34.2
//   16384x4096   64: 13.8, 64 (8 waves) 14.7, 32: 19.2  |  64: 17.7, 128 22.6, 32 26.5     |  128 (32) 24.0, 64 (32) 31.2, 128 36.2
//   18000x4096   64 (8 waves) 19.5, 64 24.8, 32: 26.1   |  128: 22.9, 64 29.5              |  128: 35.7, 128 (32) 42.5, 64 (32) 42.8
//   28672x8192   64 (8 waves) 38.7, 64 43.6, 32: 58.3   |  128: 46.0, 64 53.3              |  128: 71.7, 128 (32) 82.8, 64 (32) 98.1
// Groups of 32 under binary32 scales hold most: with 16-bit x the shapes of 2 x 8 and 8 x 2 waves (32 rows of weights, 16 of x; 128, 64) spill 8 to 10 of
// their 128 registers.
template <typename X, typename S, int GROUP> static gq_status matvec_of_group(MatvecArgs p, hipStream_t stream)
{
    const int64_t tiles = (p.rows + 15) / 16;
    if (p.m <= 8) {
        p.row_shift = 11;                                                          // whole steps of 2048 columns
        while ((1 << p.row_shift) < p.cols) p.row_shift++;
        if (((int64_t)p.m << p.row_shift) * (int)sizeof(X) <= 64 * 1024)
            return tiles <= 256 ? launch_matvec<X, S, GROUP, 1, 1, 16, 1, true>(p, stream)
                   : tiles > 512 && tiles <= 1024 && p.m == 1 ? launch_matvec<X, S, GROUP, 1, 1, 4, 4, true>(p, stream)
                                                              : launch_matvec<X, S, GROUP, 1, 1, 8, 2, true>(p, stream);
    }
    const int64_t work = tiles * ((p.m + 63) / 64);                                // of more than 64 rows of x, slices of 64 or 32
    const int size = work <= 256 ? 0 : work <= 512 ? 1 : work <= 1024 ? 2 : 3;
    if (p.m <= 16)
        return size == 0   ? launch_matvec<X, S, GROUP, 1, 1, 8, 2, false>(p, stream)
               : size == 1 ? launch_matvec<X, S, GROUP, 1, 2, 8, 2, false>(p, stream)
               : size == 2 ? launch_matvec<X, S, GROUP, 1, 4, 4, 2, false>(p, stream) : launch_matvec<X, S, GROUP, 1, 4, 2, 2, false>(p, stream);
    if (p.m <= 32)
        return size == 0   ? launch_matvec<X, S, GROUP, 1, 2, 8, 2, false>(p, stream)
               : size == 1 ? launch_matvec<X, S, GROUP, 2, 2, 8, 1, false>(p, stream)
               : size == 2 ? launch_matvec<X, S, GROUP, 2, 4, 4, 2, false>(p, stream) : launch_matvec<X, S, GROUP, 2, 8, 2, 2, false>(p, stream);
    return size == 0   ? launch_matvec<X, S, GROUP, 2, 2, 8, 1, false>(p, stream)
           : size == 1 ? launch_matvec<X, S, GROUP, 2, 4, 4, 2, false>(p, stream)
           : size == 2 ? launch_matvec<X, S, GROUP, 2, 8, 2, 2, false>(p, stream) : launch_matvec<X, S, GROUP, 4, 8, 2, 2, false>(p, stream);
}

// the product for one type of activations; the arguments have been checked
template <typename X> gq_status matvec(const MatvecArgs &p, int group, int scale_dtype, hipStream_t stream)
{
    return with_scale_type(scale_dtype, [&](auto s) {
        typedef decltype(s) S;
        return group == 32 ? matvec_of_group<X, S, 32>(p, stream) : group == 64 ? matvec_of_group<X, S, 64>(p, stream) : matvec_of_group<X, S, 128>(p, stream);
    });
}

}  // namespace gq
