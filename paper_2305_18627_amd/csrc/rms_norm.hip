// Root-mean-square norm with the residual's addition, outputs in the input's type or in 8 bits, and its backward pass.
// The contract of the entry points is stated in include/gqsgd.h.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>

#include "gqsgd.h"
#include "gq_layers.hpp"

namespace gq {

// h = residual + dropout(x), y = h rstd weight, rstd = 1 / sqrt(mean(h^2) + eps): a sum over the row and a second look at it.
// A row belongs to a team of WPR waves, whose lanes hold STEPS units of eight columns each, 64 WPR units apart, from the first
// load to the last store: a row is read once.  Teams of one wave share a workgroup of four.
template <int WPR> constexpr int kTeams = WPR == 1 ? 4 : 1;
template <int WPR> constexpr int kThreads = 64 * WPR * kTeams<WPR>;

// the sum over a team, the same for all its lanes; `lds`, the team's own, is not used again before the workgroup's next barrier but one
template <int WPR, int TEAMS = 1> __device__ __forceinline__ double team_sum(double v, double *lds)
{
    v = wave_sum(v);
    if constexpr (WPR == 1) {
        return v;
    } else {
        if ((threadIdx.x & 63) == 0) lds[TEAMS > 1 ? (threadIdx.x >> 6) % WPR : threadIdx.x >> 6] = v;
        __syncthreads();
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < WPR; i++) s += lds[i];
        return s;
    }
}
template <int WPR> __device__ __forceinline__ uint32_t team_max(uint32_t v, uint32_t *lds)
{
    v = wave_max(v);
    if constexpr (WPR == 1) {
        return v;
    } else {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < WPR; i++) m = max(m, lds[i]);
        return m;
    }
}

// 1 / sqrt(v) to about 2^-45: the instruction's estimate (2^29 units in the last place of binary64 at most, 2^-23) and one step of Newton's method
__device__ __forceinline__ float reciprocal_root(double v)
{
    const double y = __builtin_amdgcn_rsq(v);
    return v <= 1e300 ? (float)(y * (1.5 - 0.5 * v * y * y)) : (float)y;      // of an infinity: 0, which the step would make a NaN
}

struct RowScale { float scale, inv; };
// scale and what codes are multiplied by, for a row whose largest magnitude has the bits `top_bits`; per_top: 1 / the largest code
__device__ __forceinline__ RowScale row_scale(uint32_t top_bits, float per_top)
{
    const float a = __uint_as_float(top_bits);
    if (top_bits >= 0x7F800000u) return {__builtin_nanf(""), 0.0f};
    const float scale = a * per_top, inv = 1.0f / scale;
    if (!(inv <= 3.402823466e+38f)) return {0.0f, 0.0f};              // a row of zeros, or too small to be scaled
    return {scale, inv};
}

// y inv as a code; a row that is not finite has inv = 0 and gives codes 0 whatever y is
__device__ __forceinline__ float code_of(float y, float inv, float top)
{
    return inv == 0.0f ? 0.0f : __builtin_amdgcn_fmed3f(y * inv, -top, top);
}

struct NormArgs {
    const void *x, *residual, *weight;
    void *sum_out, *out;
    float *scales_out, *rstd_out;
    int64_t rows;
    int n, units;                  // units of eight columns a row
    double per_n, eps;             // 1 / n
    int draws, out_dtype;          // random bits an element, 0: no dropout
    Drop drop;
};

// Bound by memory in long launches: 8192x4096 bf16 with a residual and dropout, sum and y written, 45 us, 6.0 TB/s; fp32 without dropout
// 96 us, 5.6 TB/s.  By latency (the load, the sum's round through the team, the 8-bit maximum's) in short ones: 1x4096 2.2 us, to int8 2.6.
template <typename T, typename W, int WPR, int STEPS, bool TINY, bool RESIDUAL>
__global__ void __launch_bounds__(kThreads<WPR>)
rms_norm_kernel(NormArgs p)
{
    __shared__ double sums[WPR];
    __shared__ uint32_t tops[WPR];
    constexpr int kLanes = 64 * WPR;
    const int lane = threadIdx.x % kLanes;
    const int64_t row = (int64_t)blockIdx.x * kTeams<WPR> + threadIdx.x / kLanes;
    if (WPR == 1 && row >= p.rows) return;                            // whole waves; there is no barrier in them
    const T *x = (const T *)p.x + row * p.n, *residual = (const T *)p.residual + row * p.n;
    const W *weight = (const W *)p.weight;

    Eight<T> xr[STEPS], rr[STEPS];
    Eight<W> w[STEPS];
#pragma unroll
    for (int k = 0; k < STEPS; k++) {
        ask8<true, TINY>(x, p.n, 8 * (lane + k * kLanes), xr[k]);
        if (RESIDUAL) ask8<true, TINY>(residual, p.n, 8 * (lane + k * kLanes), rr[k]);
    }
#pragma unroll
    for (int k = 0; k < STEPS; k++) ask8<false, TINY>(weight, p.n, 8 * (lane + k * kLanes), w[k]);
    float h[STEPS][8];
    double ss = 0.0;
#pragma unroll
    for (int k = 0; k < STEPS; k++) {
        const int u = lane + k * kLanes;
        settle8<TINY>(p.n, 8 * u, xr[k]);
        if (RESIDUAL) settle8<TINY>(p.n, 8 * u, rr[k]);
#pragma unroll
        for (int i = 0; i < 8; i++) h[k][i] = xr[k].f(i);
        const uint64_t g = p.drop.first + 8 * ((uint64_t)row * p.units + u);
        if (p.draws == 32) drop8<false>(p.drop, g, h[k]);
        if (p.draws == 16) drop8<true>(p.drop, g, h[k]);
        if (RESIDUAL) {
#pragma unroll
            for (int i = 0; i < 8; i++) h[k][i] = rr[k].f(i) + h[k][i];
        }
#pragma unroll
        for (int i = 0; i < 8; i++) ss = __builtin_fma((double)h[k][i], (double)h[k][i], ss);    // zeros past the row's end
    }
    ss = team_sum<WPR>(ss, sums);
    const float rstd = reciprocal_root(__builtin_fma(ss, p.per_n, p.eps));
    if (p.rstd_out && lane == 0) p.rstd_out[row] = rstd;
    if (p.sum_out) {
#pragma unroll
        for (int k = 0; k < STEPS; k++) store8((T *)p.sum_out + row * p.n + 8 * (lane + k * kLanes), p.n - 8 * (lane + k * kLanes), h[k]);
    }
#pragma unroll
    for (int k = 0; k < STEPS; k++) {
        settle8<TINY>(p.n, 8 * (lane + k * kLanes), w[k]);
#pragma unroll
        for (int i = 0; i < 8; i++) h[k][i] = (h[k][i] * rstd) * w[k].f(i);
    }
    if (!p.scales_out) {
#pragma unroll
        for (int k = 0; k < STEPS; k++) store8((T *)p.out + row * p.n + 8 * (lane + k * kLanes), p.n - 8 * (lane + k * kLanes), h[k]);
        return;
    }
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < STEPS; k++)
#pragma unroll
        for (int i = 0; i < 8; i++) m = max(m, 8 * (lane + k * kLanes) + i < p.n ? __float_as_uint(h[k][i]) & 0x7FFFFFFFu : 0u);
    const float top = p.out_dtype == GQ_I8 ? 127.0f : 448.0f;
    const RowScale rs = row_scale(team_max<WPR>(m, tops), p.out_dtype == GQ_I8 ? 1.0f / 127.0f : 1.0f / 448.0f);
    if (lane == 0) p.scales_out[row] = rs.scale;
#pragma unroll
    for (int k = 0; k < STEPS; k++) {
        float c[8];
        struct { uint8_t e[8]; } o;
#pragma unroll
        for (int i = 0; i < 8; i++) c[i] = code_of(h[k][i], rs.inv, top);
        if (p.out_dtype == GQ_I8) {
#pragma unroll
            for (int i = 0; i < 8; i++) o.e[i] = (uint8_t)(int8_t)(int)__builtin_rintf(c[i]);
        } else {
            u32x2 v = {0u, 0u};
#pragma unroll
            for (int i = 0; i < 2; i++) {
                v[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[4 * i], c[4 * i + 1], 0, false);
                v[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[4 * i + 2], c[4 * i + 3], (int)v[i], true);
            }
            __builtin_memcpy(&o, &v, 8);
        }
        const int u = lane + k * kLanes, left = p.n - 8 * u;
        uint8_t *at = (uint8_t *)p.out + row * p.n + 8 * u;
        if (left >= 8) {
            __builtin_memcpy(at, &o, 8);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (i < left) at[i] = o.e[i];
        }
    }
}

struct BackwardArgs {
    const void *dy, *h, *dsum, *weight;
    const float *rstd;
    void *dres_out, *dx_out;
    float *parts;                  // [teams' workgroups][8 units], or NULL
    int64_t rows;
    int n, units;
    double per_n;
    int draws;
    Drop drop;
};

// the compiler may not keep what it computed from these before
template <typename T> __device__ __forceinline__ void forget(Eight<T> &t)
{
#pragma unroll
    for (size_t i = 0; i < sizeof(t) / 4; i++) {
        uint32_t w = t.w[i];
        asm volatile("" : "+v"(w));
        t.w[i] = w;
    }
}

__device__ __forceinline__ void store_part(float *part, const double *dw)
{
#pragma unroll
    for (int i = 0; i < 8; i += 4) *reinterpret_cast<f32x4 *>(part + i) = f32x4{(float)dw[i], (float)dw[i + 1], (float)dw[i + 2], (float)dw[i + 3]};
}

// dh = dsum + rstd (g - xh mean(g xh)) and dweight = sum over rows of dy xh, with xh = h rstd, g = dy weight: one pass over the rows.
// A workgroup takes rows (its teams one each) in turn, gridDim.x * teams apart, and keeps the weight's gradient of its columns in
// registers; its sums go to `parts` and a second kernel adds those up.  AHEAD: the next row is asked for before the current one is
// reduced, where the registers reach.  dweight is summed in binary64, where the products are exact, and rounded once a part and once at the
// end, so that its error does not grow with the rows; sums in binary32 are no faster (8192x4096 bf16 40.5 us with both).
// Bound by memory: 8192x4096 bf16 with dsum and dropout 61 us, 5.5 TB/s, and 4.8 us for the parts' sum; 1000x2047 fp32, four rows a
// workgroup one after another, 8.4 and 2.5 us.
template <typename T, typename W, int WPR, int STEPS, int TEAMS, bool TINY, bool DSUM, bool AHEAD>
__global__ void __launch_bounds__(64 * WPR * TEAMS)
rms_norm_backward_kernel(BackwardArgs p)
{
    constexpr int kLanes = 64 * WPR, kTeam = TEAMS;
    constexpr bool kTogether = TEAMS > 1 && WPR > 1;                  // there is a barrier in each turn, and several teams at it
    __shared__ double sums[2][kTeam][WPR];
    __shared__ double joined[kTeam > 1 ? kTeam - 1 : 1][kTeam > 1 ? STEPS * 8 * kLanes : 1];
    const int lane = threadIdx.x % kLanes, team = threadIdx.x / kLanes;
    const int64_t stride = (int64_t)gridDim.x * kTeam;
    struct Row { Eight<T> dy[STEPS], h[STEPS], ds[DSUM ? STEPS : 1]; float rstd; };
    auto fetch = [&](int64_t row, Row &r) {
        r.rstd = p.rstd[row];
#pragma unroll
        for (int k = 0; k < STEPS; k++) {
            const int c = 8 * (lane + k * kLanes);
            ask8<true, TINY>((const T *)p.dy + row * p.n, p.n, c, r.dy[k]);
            ask8<true, TINY>((const T *)p.h + row * p.n, p.n, c, r.h[k]);
            if (DSUM) ask8<true, TINY>((const T *)p.dsum + row * p.n, p.n, c, r.ds[k]);
        }
    };
    Eight<W> w[STEPS];
    Row now, next;
    double dw[STEPS][8];
#pragma unroll
    for (int k = 0; k < STEPS; k++) {
        ask8<false, TINY>((const W *)p.weight, p.n, 8 * (lane + k * kLanes), w[k]);
        settle8<TINY>(p.n, 8 * (lane + k * kLanes), w[k]);
#pragma unroll
        for (int i = 0; i < 8; i++) dw[k][i] = 0.0;
    }
    int64_t row = (int64_t)blockIdx.x * kTeam + team;
    if (AHEAD && row < p.rows) fetch(row, now);
    // at a barrier as many turns for each team: one without a row only takes part in that
    for (int turn = 0; (kTogether ? row - team : row) < p.rows; row += stride, turn ^= 1) {
        const bool live = !kTogether || row < p.rows;
        if (!AHEAD && live) fetch(row, now);
        if (AHEAD && row + stride < p.rows) fetch(row + stride, next);
        const float rstd = now.rstd;
        double s = 0.0;
#pragma unroll
        for (int k = 0; k < STEPS && live; k++) {
            settle8<TINY>(p.n, 8 * (lane + k * kLanes), now.dy[k]);
            settle8<TINY>(p.n, 8 * (lane + k * kLanes), now.h[k]);
            if (DSUM) settle8<TINY>(p.n, 8 * (lane + k * kLanes), now.ds[k]);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float dy = now.dy[k].f(i), xh = now.h[k].f(i) * rstd;
                s = __builtin_fma((double)(dy * w[k].f(i)), (double)xh, s);
                dw[k][i] = __builtin_fma((double)dy, (double)xh, dw[k][i]);
            }
            __builtin_amdgcn_sched_barrier(0);                        // a unit after another: all at once hold too many registers
        }
        const float mean = (float)(team_sum<WPR, kTeam>(s, sums[turn][team]) * p.per_n);
#pragma unroll
        for (int k = 0; k < STEPS && live; k++) {
            const int u = lane + k * kLanes, left = p.n - 8 * u;
            const int64_t at = row * p.n + 8 * u;
            forget(now.dy[k]);
            forget(now.h[k]);
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float g = now.dy[k].f(i) * w[k].f(i), xh = now.h[k].f(i) * rstd;
                v[i] = rstd * (g - xh * mean);
                if (DSUM) v[i] = now.ds[k].f(i) + v[i];
            }
            if (p.dres_out) store8((T *)p.dres_out + at, left, v);
            const uint64_t g = p.drop.first + 8 * ((uint64_t)row * p.units + u);
            if (p.draws == 32) drop8<false>(p.drop, g, v);
            if (p.draws == 16) drop8<true>(p.drop, g, v);
            store8((T *)p.dx_out + at, left, v);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (AHEAD) now = next;
    }
    if (!p.parts) return;
    if (kTeam > 1) {
        if (team > 0) {
#pragma unroll
            for (int k = 0; k < STEPS; k++)
#pragma unroll
                for (int i = 0; i < 8; i++) joined[team - 1][(k * 8 + i) * kLanes + lane] = dw[k][i];
        }
        __syncthreads();
        if (team > 0) return;
#pragma unroll
        for (int t = 0; t < kTeam - 1; t++)
#pragma unroll
            for (int k = 0; k < STEPS; k++)
#pragma unroll
                for (int i = 0; i < 8; i++) dw[k][i] += joined[t][(k * 8 + i) * kLanes + lane];
    }
    float *part = p.parts + (int64_t)blockIdx.x * p.units * 8;
#pragma unroll
    for (int k = 0; k < STEPS; k++) {
        const int u = lane + k * kLanes;
        if (u < p.units) {
            store_part(part + 8 * u, dw[k]);
        }
    }
}

// The same for rows that the registers of a team do not hold beside the weight's gradient: dy and h stay in LDS from the first look at a row to
// the second, 128 KB for STEPS units a lane; dy alone where that is not enough (binary32 above 16384 columns: h is read again).
// Bound by memory and what a step does not overlap: with dsum 1024x32768 bf16 66.6 us, 4.0 TB/s (75.8 with each row read twice), fp32 135, 4.0;
// 4096x16384 bf16 102, 5.3, without dsum 85, 4.7.
constexpr int kLongBlock = 1024;
constexpr int kLongLds = 128 * 1024;
template <typename T, typename W, int STEPS>
__global__ void __launch_bounds__(kLongBlock)
rms_norm_backward_long_kernel(BackwardArgs p)
{
    constexpr int kWaves = kLongBlock / 64, kChunks = sizeof(T) / 2;           // of 16 bytes a unit
    constexpr bool kKeepH = 2 * STEPS * kChunks * 16 * kLongBlock <= kLongLds;
    constexpr int kPer = kKeepH ? 2 * kChunks : kChunks;
    static_assert(STEPS * kPer * 16 * kLongBlock <= kLongLds, "LDS");
    extern __shared__ u32x4 kept[];                                            // [STEPS][kPer][lanes], each touched by one lane only
    __shared__ double sums[2][kWaves];
    const int first = __builtin_amdgcn_readfirstlane(threadIdx.x & ~63);       // the wave's first unit
    auto keep = [&](int at, const Eight<T> &t) {
#pragma unroll
        for (int i = 0; i < kChunks; i++) kept[(at + i) * kLongBlock + threadIdx.x] = u32x4{t.w[4 * i], t.w[4 * i + 1], t.w[4 * i + 2], t.w[4 * i + 3]};
    };
    auto recall = [&](int at, Eight<T> &t) {
#pragma unroll
        for (int i = 0; i < kChunks; i++) {
            const u32x4 v = kept[(at + i) * kLongBlock + threadIdx.x];
#pragma unroll
            for (int j = 0; j < 4; j++) t.w[4 * i + j] = v[j];
        }
    };
    // as far as the registers reach: the next row's units asked for when the current one's are in LDS, and the weight held
    constexpr bool kAhead = STEPS == 2, kHoldW = STEPS == 2 && sizeof(T) == 2;
    constexpr int kHeld = kAhead ? STEPS : 1;
    Eight<T> a[kHeld], b[kHeld];
    Eight<W> w[kHoldW ? STEPS : 1];
    double dw[STEPS][8];
    int turn = 0, t = threadIdx.x;
#pragma unroll
    for (int k = 0; k < STEPS; k++) {
        if (kHoldW) {
            ask8<false, false>((const W *)p.weight, p.n, 8 * (t + k * kLongBlock), w[kHoldW ? k : 0]);
            settle8<false>(p.n, 8 * (t + k * kLongBlock), w[kHoldW ? k : 0]);
        }
#pragma unroll
        for (int i = 0; i < 8; i++) dw[k][i] = 0.0;
    }
    auto ask_row = [&](int64_t row) {
#pragma unroll
        for (int k = 0; k < kHeld; k++) {
            ask8<true, false>((const T *)p.dy + row * p.n, p.n, 8 * (t + k * kLongBlock), a[k]);
            ask8<kKeepH, false>((const T *)p.h + row * p.n, p.n, 8 * (t + k * kLongBlock), b[k]);
        }
    };
    if (kAhead && blockIdx.x < p.rows) ask_row(blockIdx.x);
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1) {
        asm volatile("" : "+v"(t));                                             // addresses are formed in each row, not held
        const float rstd = p.rstd[row];
        const T *dy = (const T *)p.dy + row * p.n, *h = (const T *)p.h + row * p.n;
        double s = 0.0;
#pragma unroll
        for (int k = 0; k < STEPS; k++) {
            if (first + k * kLongBlock >= p.units) continue;                    // the whole wave
            const int c = 8 * (t + k * kLongBlock), at = kAhead ? k : 0, wk = kHoldW ? k : 0;
            if (kHoldW) forget(w[wk]);
            else ask8<false, false>((const W *)p.weight, p.n, c, w[wk]);
            if (!kAhead) {
                ask8<true, false>(dy, p.n, c, a[at]);
                ask8<kKeepH, false>(h, p.n, c, b[at]);
            }
            settle8<false>(p.n, c, a[at]);
            settle8<false>(p.n, c, b[at]);
            if (!kHoldW) settle8<false>(p.n, c, w[wk]);
            keep(k * kPer, a[at]);
            if (kKeepH) keep(k * kPer + kChunks, b[at]);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float xh = b[at].f(i) * rstd;
                s = __builtin_fma((double)(a[at].f(i) * w[wk].f(i)), (double)xh, s);
                dw[k][i] = __builtin_fma((double)a[at].f(i), (double)xh, dw[k][i]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (kAhead) ask_row(min(row + (int64_t)gridDim.x, p.rows - 1));        // past the last row that one again, not used
        const float mean = (float)(team_sum<kWaves>(s, sums[turn]) * p.per_n);
        auto second = [&](int k, Eight<W> &w) {
            const int u = t + k * kLongBlock, left = p.n - 8 * u;
            Eight<T> y, x, ds;
            if (!kKeepH) ask8<true, false>(h, p.n, 8 * u, x);
            if (kHoldW) forget(w);
            else ask8<false, false>((const W *)p.weight, p.n, 8 * u, w);
            if (p.dsum) ask8<true, false>((const T *)p.dsum + row * p.n, p.n, 8 * u, ds);
            recall(k * kPer, y);
            if (kKeepH) recall(k * kPer + kChunks, x);
            else settle8<false>(p.n, 8 * u, x);
            if (!kHoldW) settle8<false>(p.n, 8 * u, w);
            if (p.dsum) settle8<false>(p.n, 8 * u, ds);
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                v[i] = rstd * (y.f(i) * w.f(i) - (x.f(i) * rstd) * mean);
                if (p.dsum) v[i] = ds.f(i) + v[i];
            }
            if (p.dres_out) store8((T *)p.dres_out + row * p.n + 8 * u, left, v);
            const uint64_t g = p.drop.first + 8 * ((uint64_t)row * p.units + u);
            if (p.draws == 32) drop8<false>(p.drop, g, v);
            if (p.draws == 16) drop8<true>(p.drop, g, v);
            store8((T *)p.dx_out + row * p.n + 8 * u, left, v);
        };
        if (kHoldW) {
#pragma unroll
            for (int k = 0; k < STEPS; k++)
                if (first + k * kLongBlock < p.units) second(k, w[kHoldW ? k : 0]);
        } else {
#pragma unroll 1
            for (int k = 0; k < STEPS && first + k * kLongBlock < p.units; k++) second(k, w[0]);
        }
    }
    if (!p.parts) return;
    float *part = p.parts + (int64_t)blockIdx.x * p.units * 8;
#pragma unroll
    for (int k = 0; k < STEPS; k++) {
        const int u = threadIdx.x + k * kLongBlock;
        if (u < p.units) store_part(part + 8 * u, dw[k]);
    }
}

// A workgroup adds up `count` parts of kSumColumns columns: a lane four columns of a slice of the parts, joined in a fixed order.
// 32: 2048x2048 12.5 us with the whole backward pass, 64: 13.0, 16: 13.4; 1000x2047 13.7, 14.1, 12.7
constexpr int kSumColumns = 32, kSumLanes = kSumColumns / 4, kSlices = 256 / kSumLanes;
__global__ void __launch_bounds__(256)
weight_sum_kernel(const float *parts, int count, int n, int pitch, float *dweight)
{
    __shared__ double slices[kSlices][kSumColumns];
    const int c4 = threadIdx.x % kSumLanes, slice = threadIdx.x / kSumLanes, c = blockIdx.x * kSumColumns + 4 * c4;
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    const float *from = parts + (c < pitch ? c : 0);
    for (int i = slice; i < count; i += 8 * kSlices) {
        f32x4 v[8];                                                            // asked for together
#pragma unroll
        for (int k = 0; k < 8; k++) v[k] = *reinterpret_cast<const f32x4 *>(from + (int64_t)min(i + k * kSlices, count - 1) * pitch);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < 8; k++)
#pragma unroll
            for (int j = 0; j < 4; j++) s[j] += i + k * kSlices < count ? (double)v[k][j] : 0.0;
    }
#pragma unroll
    for (int j = 0; j < 4; j++) slices[slice][4 * c4 + j] = s[j];
    __syncthreads();
    const int column = blockIdx.x * kSumColumns + threadIdx.x;
    if (threadIdx.x >= kSumColumns || column >= n) return;
    double t = 0.0;
#pragma unroll
    for (int i = 0; i < kSlices; i++) t += slices[i][threadIdx.x];
    dweight[column] = (float)t;
}

static gq_status check_norm(int64_t rows, int64_t n, int dtype, int weight_dtype, const gq_dropout_params *drop)
{
    if (!float_type(dtype) || (weight_dtype != GQ_F32 && weight_dtype != dtype) || !matrix_fits(rows, n)) return GQ_ERR_INVALID_ARG;
    if (drop && check_drop(drop, rows, n) != GQ_OK) return GQ_ERR_INVALID_ARG;
    return n > GQ_RMS_NORM_MAX_N ? GQ_ERR_UNSUPPORTED : GQ_OK;
}
static int draw_bits(const gq_dropout_params *p) { return !p ? 0 : short_draws(p) ? 16 : 32; }

template <typename F> static gq_status with_types(int dtype, int weight_dtype, F &&f)
{
    return with_float_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return weight_dtype == GQ_F32 ? f(t, float()) : f(t, T());
    });
}

// f(waves per row, steps, fewer than eight columns) of the smallest team that holds a row of n columns, as compile-time constants.  Of
// up to kFewRows rows, less than what a unit's latency covers, with one step a lane: 61x5003 fp16 to 8 bits 4.8 and 4.7 us, 1x4096
// 2.9, 2.7, 64x8192 fp32 with dropout 5.9, 4.8, 256x8192 bf16 4.7, 4.7; 8192 rows of 4096 columns have one of 4 waves (45 us).
constexpr int64_t kFewRows = 256;
template <typename F> static gq_status with_team(int64_t rows, int64_t n, F &&f)
{
    using std::integral_constant;
    const std::false_type no;
    if (n < 8) return f(integral_constant<int, 1>(), integral_constant<int, 1>(), std::true_type());
    if (rows <= kFewRows && n > 2048 && n <= 4096) return f(integral_constant<int, 8>(), integral_constant<int, 1>(), no);
    if (rows <= kFewRows && n > 4096 && n <= 8192) return f(integral_constant<int, 16>(), integral_constant<int, 1>(), no);
    if (n <= 512) return f(integral_constant<int, 1>(), integral_constant<int, 1>(), no);
    if (n <= 1024) return f(integral_constant<int, 1>(), integral_constant<int, 2>(), no);
    if (n <= 2048) return f(integral_constant<int, 4>(), integral_constant<int, 1>(), no);
    if (n <= 4096) return f(integral_constant<int, 4>(), integral_constant<int, 2>(), no);
    if (n <= 6144) return f(integral_constant<int, 4>(), integral_constant<int, 3>(), no);
    if (n <= 8192) return f(integral_constant<int, 4>(), integral_constant<int, 4>(), no);
    if (n <= 16384) return f(integral_constant<int, 16>(), integral_constant<int, 2>(), no);
    return f(integral_constant<int, 16>(), integral_constant<int, 4>(), no);
}

constexpr int64_t kManyRows = 2048;
constexpr int64_t kMostHeld = 8192;       // columns that the registers of a team hold in the backward pass
static bool four_teams(int64_t rows, int64_t n) { return n > 1024 && n <= 2048 && rows >= kManyRows; }

// f(waves per row, steps, teams a workgroup, fewer than eight columns) for the backward pass, whose rows come with twice the registers;
// for rows of up to kMostHeld columns.  Above 6144 columns 16 waves of one step and 8 of two take: 8192x8192 bf16 74.3 and 77.8 us, with dropout
// 117 and 139, with dsum 93 and 90; 4096x7000 41 and 50.  Teams of four waves: one a workgroup for few rows, four, with one part of the weight's
// gradient between them, for many.  us with one and four: 300x2047 bf16 7.7, 8.5; 1000x2047 fp32 11.1, 13.7;
// 1500x2047 13.5, 15.6, 2048x2047 17.3, 17.6; bf16 4096x2047 22.8, 18.4; with dropout 2048x2048 15.9, 12.5, 16384x2048 70.5, 61.3.
template <typename F> static gq_status with_backward_team(int64_t rows, int64_t n, F &&f)
{
    using std::integral_constant;
    const std::false_type no;
    const integral_constant<int, 1> one;
    const integral_constant<int, 4> four;
    if (n < 8) return f(integral_constant<int, 1>(), integral_constant<int, 1>(), four, std::true_type());
    if (n <= 512) return f(integral_constant<int, 1>(), integral_constant<int, 1>(), four, no);
    if (n <= 1024) return f(integral_constant<int, 1>(), integral_constant<int, 2>(), four, no);
    if (n <= 2048) return four_teams(rows, n) ? f(four, one, four, no) : f(four, one, one, no);
    if (n <= 4096) return f(integral_constant<int, 8>(), integral_constant<int, 1>(), one, no);
    if (n <= 6144) return f(integral_constant<int, 12>(), integral_constant<int, 1>(), one, no);
    return f(integral_constant<int, 16>(), one, one, no);
}

// Workgroups of the backward pass, each of which leaves one part of the weight's gradient: one a compute unit where it has enough
// waves of its own and asks ahead, else two.  bf16, us with 256 and 512: 8192x4096 47.8 and 51.8, with dropout (more arithmetic, and
// no asking ahead) 71.6 and 64.0, but of 12 waves, of which two no longer fit, 8192x6000 95 and 112; of one team of four waves each
// 1000x2047 fp32 11.3 and 12.0: too few rows each to make up for the parts.
constexpr int64_t kMostParts = 512;
static int64_t backward_groups(int64_t rows, int64_t n, bool drop)
{
    const int64_t teams = n <= 1024 || four_teams(rows, n) ? (rows + 3) / 4 : rows;
    const bool two = (n <= 512 || (drop && n <= 4096 && (n <= 1024 || n > 2048))) && teams >= 4 * kMostParts;
    const int64_t most = two ? kMostParts : kMostParts / 2;
    return teams < 1 ? 1 : teams < most ? teams : most;
}

}  // namespace gq

using namespace gq;

extern "C" {

gq_status gq_rms_norm(const void *x, const void *residual, int64_t rows, int64_t n, gq_dtype dtype, const void *weight,
                      gq_dtype weight_dtype, float eps, const gq_dropout_params *drop, void *sum_out, void *out, gq_dtype out_dtype,
                      float *scales_out, float *rstd_out, void *hip_stream)
{
    const gq_status st = check_norm(rows, n, dtype, weight_dtype, drop);
    if (st != GQ_OK) return st;
    const bool bytes = out_dtype == GQ_I8 || out_dtype == GQ_E4M3;
    if (!(eps > 0.0f && eps <= 3.402823466e+38f) || (!bytes && out_dtype != dtype) || bytes != (scales_out != nullptr)) return GQ_ERR_INVALID_ARG;
    if (rows == 0 || n == 0) return GQ_OK;
    if (!aligned(x, 16) || !aligned(weight, 16) || !aligned(out, 16) || !aligned_or_null(residual, 16) || !aligned_or_null(sum_out, 16) ||
        !aligned_or_null(scales_out, 4) || !aligned_or_null(rstd_out, 4) || out == sum_out) return GQ_ERR_INVALID_ARG;
    if (bytes && (out == x || out == residual)) return GQ_ERR_INVALID_ARG;         // rows of codes lie over other rows of the input
    const NormArgs p = {x, residual, weight, sum_out, out, scales_out, rstd_out, rows, (int)n, (int)(pitch8(n) / 8), 1.0 / (double)n, (double)eps,
                        draw_bits(drop), (int)out_dtype, drop ? make_drop(drop) : Drop{}};
    return with_types(dtype, weight_dtype, [&](auto t, auto w) {
        typedef decltype(t) T;
        typedef decltype(w) W;
        return with_team(rows, n, [&](auto wpr, auto steps, auto tiny) {
            constexpr int WPR = decltype(wpr)::value, STEPS = decltype(steps)::value;
            constexpr bool TINY = decltype(tiny)::value;
            const int64_t blocks = (rows + kTeams<WPR> - 1) / kTeams<WPR>;
            if (!grid_fits(blocks, kThreads<WPR>)) return GQ_ERR_INVALID_ARG;
            auto kernel = residual ? rms_norm_kernel<T, W, WPR, STEPS, TINY, true> : rms_norm_kernel<T, W, WPR, STEPS, TINY, false>;
            kernel<<<(unsigned)blocks, kThreads<WPR>, 0, (hipStream_t)hip_stream>>>(p);
            return launched();
        });
    });
}

size_t gq_rms_norm_workspace_bytes(int64_t rows, int64_t n)
{
    if (!matrix_fits(rows, n) || n > GQ_RMS_NORM_MAX_N) return 0;
    return (size_t)((rows < 1 ? 1 : rows < kMostParts ? rows : kMostParts) * pitch8(n) * 4);
}

gq_status gq_rms_norm_backward(const void *dy, const void *h, const void *dsum, int64_t rows, int64_t n, gq_dtype dtype,
                               const void *weight, gq_dtype weight_dtype, const float *rstd, const gq_dropout_params *drop, void *dres_out,
                               void *dx_out, float *dweight_out, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const gq_status st = check_norm(rows, n, dtype, weight_dtype, drop);
    if (st != GQ_OK) return st;
    if (!drop && dres_out) return GQ_ERR_INVALID_ARG;
    if (n == 0 || (rows == 0 && !dweight_out)) return GQ_OK;
    if (rows > 0 && (!aligned(dy, 16) || !aligned(h, 16) || !aligned(weight, 16) || !aligned(rstd, 4) || !aligned(dx_out, 16) ||
                     !aligned_or_null(dsum, 16) || !aligned_or_null(dres_out, 16) || dres_out == dx_out)) return GQ_ERR_INVALID_ARG;
    if (!aligned_or_null(dweight_out, 16)) return GQ_ERR_INVALID_ARG;
    if (dweight_out && (!aligned(workspace, 16) || workspace_bytes < gq_rms_norm_workspace_bytes(rows, n))) return GQ_ERR_WORKSPACE;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const int64_t groups = backward_groups(rows, n, drop != nullptr);
    const BackwardArgs p = {dy, h, dsum, weight, rstd, dres_out, dx_out, dweight_out ? (float *)workspace : nullptr, rows, (int)n,
                            (int)(pitch8(n) / 8), 1.0 / (double)n, draw_bits(drop), drop ? make_drop(drop) : Drop{}};
    if (rows > 0) {
        const gq_status launch = with_types(dtype, weight_dtype, [&](auto t, auto w) {
            typedef decltype(t) T;
            typedef decltype(w) W;
            if (n > kMostHeld) {
                auto kernel = n > 2 * kMostHeld ? rms_norm_backward_long_kernel<T, W, 4> : rms_norm_backward_long_kernel<T, W, 2>;
                kernel<<<(unsigned)groups, kLongBlock, kLongLds, stream>>>(p);
                return launched();
            }
            return with_backward_team(rows, n, [&](auto wpr, auto steps, auto of, auto tiny) {
                constexpr int WPR = decltype(wpr)::value, STEPS = decltype(steps)::value, TEAMS = decltype(of)::value;
                constexpr bool TINY = decltype(tiny)::value;
                auto with_dsum = [&](auto there) {
                    constexpr bool DSUM = decltype(there)::value;
                    constexpr bool kTwo = WPR == 1 || WPR == 8;        // where there may be two workgroups a compute unit, with dropout
                    // as far as the registers reach: with the next row of binary32 and dsum, 16 waves spill (4096x8192 105.4 us, 101.5 without)
                    constexpr bool kAhead = !(WPR == 16 && DSUM && sizeof(T) == 4);
                    return kTwo && groups == kMostParts && drop ? rms_norm_backward_kernel<T, W, WPR, STEPS, TEAMS, TINY, DSUM, !kTwo && kAhead>
                                                                : rms_norm_backward_kernel<T, W, WPR, STEPS, TEAMS, TINY, DSUM, kAhead>;
                };
                auto kernel = dsum ? with_dsum(std::true_type()) : with_dsum(std::false_type());
                kernel<<<(unsigned)groups, 64 * WPR * TEAMS, 0, stream>>>(p);
                return launched();
            });
        });
        if (launch != GQ_OK) return launch;
    }
    if (!dweight_out) return GQ_OK;
    weight_sum_kernel<<<(unsigned)((n + kSumColumns - 1) / kSumColumns), 256, 0, stream>>>((const float *)workspace, rows > 0 ? (int)groups : 0, (int)n, (int)pitch8(n), dweight_out);
    return launched();
}

}  // extern "C"
