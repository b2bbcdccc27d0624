// Layer norm of n x rows rows of `width` values and its backward pass.  A row is held in registers by a team of
// L threads, E values each, from its one load to its one store: the mean is known before the squares of the distances from
// it are summed, and corrected by the distances, so a row far from zero loses nothing but what the mean's 24 bits leave out for the backward pass.  Memory
// bounds both passes.  (Where 1,024 threads hold 16 values each, 8,193 to 16,384 wide, the backward pass has too few registers for x, dy and the next row's:
// 176 bytes a thread of fp32 rows, 84 of 16-bit ones, go through scratch memory; 2 x 2,000 x 12,000 240 us and 112, 2.4 and 2.6 TB/s, forward 93 and 55.)
#pragma once
#include "layer_common.hpp"

namespace svgd {

// Sum over a team of L threads, in all of them.  Teams of more than a wave are workgroups (64 .. 1024 threads): `slots` is
// LDS of 2 * 16 floats, used by turns, so that one barrier per sum is enough.
template <int L> struct TeamSum {
    float *slots;
    int turn = 0;
    __device__ __forceinline__ float operator()(float v)
    {
        if constexpr (L <= 16) {
            return row_sum<L>(v);
        } else if constexpr (L == 32) {
            const unsigned u = __float_as_uint(row_sum(v));
            const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
            return __uint_as_float(r[0]) + __uint_as_float(r[1]);
        } else if constexpr (L == 64) {
            return wave_sum(v);
        } else {
            float *const s = slots + 16 * turn;
            turn ^= 1;
            v = wave_sum(v);
            if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
            __syncthreads();
            v = 0.f;
#pragma unroll
            for (int w = 0; w < L / 64; ++w) v += s[w];
            return v;
        }
    }
};

template <int L> constexpr int kTeamBlock = L > 256 ? L : 256; // threads per workgroup
template <int L> constexpr int kTeams = kTeamBlock<L> / L;     // rows at a time

struct NormShape {
    int64_t rows;
    int width;
    int blocks;       // workgroups per particle
    int64_t per;      // rows of each
};
template <class T> struct ActRows {
    T *p;
    int64_t particle, row;
};

// A thread's part of a row, as it comes from memory; packs beyond the width (`left` of the first pack on) count as 0.
template <class T, int L, int E> struct RowPart {
    static constexpr int VEC = 16 / sizeof(T), C = E / VEC;
    typename Pack<T, VEC>::raw v[C];
    __device__ __forceinline__ void load(const T *row, int lane, int width)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * L + lane) * VEC;
            if (col + VEC <= width) {
                v[c] = *reinterpret_cast<const typename Pack<T, VEC>::type *>(row + col);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    v[c][e] = (T)0.f;
                    if (col + e < width) v[c][e] = row[col + e];
                }
            }
        }
    }
    __device__ __forceinline__ float operator()(int c, int e) const { return (float)v[c][e]; }
};

template <class T, int L, int E>
__global__ __launch_bounds__(kTeamBlock<L>) void norm_forward_kernel(NormShape s, ActRows<const T> x, Params weight, Params bias, float eps, ActRows<T> y,
                                                                     float *mean_out, float *rstd_out)
{
    constexpr int VEC = 16 / sizeof(T), C = E / VEC;
    __shared__ float slots[32];
    TeamSum<L> sum{slots};
    const int lane = threadIdx.x % L, team = threadIdx.x / L;
    const int64_t particle = blockIdx.x / s.blocks;
    const int64_t first = (blockIdx.x % s.blocks) * s.per, last = first + s.per < s.rows ? first + s.per : s.rows;
    float w[E], b[E];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * L + lane) * VEC;
        float v[VEC];
        load_pack<float, VEC>(weight.p + particle * weight.stride + col, s.width - col, v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[c * VEC + e] = v[e];
        load_pack<float, VEC>(bias.p + particle * bias.stride + col, bias.p ? s.width - col : 0, v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) b[c * VEC + e] = v[e];
    }
    const float inv = 1.f / (float)s.width;
    RowPart<T, L, E> next; // the next row is on its way while one is worked on
    const T *const rows = x.p + particle * x.particle;
    next.load(rows + (first + team) * x.row, lane, first + team < last ? s.width : 0);
    for (int64_t r0 = first; r0 < last; r0 += kTeams<L>) {
        const int64_t r = r0 + team;
        const bool live = r < last;
        float v[C][VEC], total = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                v[c][e] = next(c, e);
                total += v[c][e];
            }
        if (r0 + kTeams<L> < last) next.load(rows + (r + kTeams<L>) * x.row, lane, r + kTeams<L> < last ? s.width : 0);
        const float mean = sum(total) * inv;
        float square = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                v[c][e] -= mean;
                if ((c * L + lane) * VEC + e < s.width) square += v[c][e] * v[c][e];
            }
        float variance = sum(square) * inv, rest = 0.f;
        // The sum's roundings put the mean off by some 2^-21 of it: nothing, unless the row is far from zero by its spread.  Then what is
        // left of the mean is found among the distances (taken with every row: 8 x 1,576 x 384 bf16 9.0 us, so 8.6).  A team's threads have the same
        // bits here, so they go the same way.
        if (mean * mean > 16.f * (variance + eps)) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if ((c * L + lane) * VEC + e < s.width) rest += v[c][e];
            rest = sum(rest) * inv;
            variance -= rest * rest;
            variance = variance < 0.f ? 0.f : variance; // (of a row of equal values)
        }
        const float rstd = 1.f / sqrtf(variance + eps);
        if (!live) continue;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * L + lane) * VEC;
            float out[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) out[e] = (v[c][e] - rest) * rstd * w[c * VEC + e] + b[c * VEC + e];
            store_pack<T, VEC>(y.p + particle * y.particle + r * y.row + col, s.width - col, out);
        }
        if (lane == 0) {
            if (mean_out) mean_out[particle * s.rows + r] = mean + rest;
            if (rstd_out) rstd_out[particle * s.rows + r] = rstd;
        }
    }
}

// dx row by row; every thread adds up dy xhat and dy of its columns over the workgroup's rows, the teams' sums are added
// in LDS and go to partials[workgroup][2][width].  norm_reduce_kernel adds those: no atomics, the same bits every time.
template <class T, int L, int E>
__global__ __launch_bounds__(kTeamBlock<L>) void norm_backward_kernel(NormShape s, ActRows<const T> dy, ActRows<const T> x, Params weight,
                                                                      const float *mean_in, const float *rstd_in, ActRows<T> dx, float *partials)
{
    constexpr int VEC = 16 / sizeof(T), C = E / VEC;
    __shared__ float slots[32];
    __shared__ float sums[kTeams<L> > 1 ? 2 * E * kTeamBlock<L> : 1];
    TeamSum<L> sum{slots};
    const int lane = threadIdx.x % L, team = threadIdx.x / L;
    const int64_t particle = blockIdx.x / s.blocks;
    const int64_t first = (blockIdx.x % s.blocks) * s.per, last = first + s.per < s.rows ? first + s.per : s.rows;
    float w[C][VEC], dw[C][VEC], db[C][VEC];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * L + lane) * VEC;
        load_pack<float, VEC>(weight.p + particle * weight.stride + col, s.width - col, w[c]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) dw[c][e] = db[c][e] = 0.f;
    }
    const float inv = 1.f / (float)s.width;
    RowPart<T, L, E> next_x, next_d; // the next row is on its way while one is worked on
    float next_mean, next_rstd;
    const auto fetch = [&](int64_t r) {
        const bool live = r < last;
        next_x.load(x.p + particle * x.particle + r * x.row, lane, live ? s.width : 0);
        next_d.load(dy.p + particle * dy.particle + r * dy.row, lane, live ? s.width : 0);
        next_mean = live ? mean_in[particle * s.rows + r] : 0.f;
        next_rstd = live ? rstd_in[particle * s.rows + r] : 0.f;
    };
    fetch(first + team);
    for (int64_t r0 = first; r0 < last; r0 += kTeams<L>) {
        const int64_t r = r0 + team;
        const bool live = r < last;
        const float mean = next_mean, rstd = next_rstd;
        float v[C][VEC], d[C][VEC], sa = 0.f, sax = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                v[c][e] = next_x(c, e);
                d[c][e] = next_d(c, e);
            }
        if (r0 + kTeams<L> < last) fetch(r + kTeams<L>);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) { // (beyond the width dy and weight are 0; x is not to count either: -mean * rstd may be infinite)
                v[c][e] = (c * L + lane) * VEC + e < s.width ? (v[c][e] - mean) * rstd : 0.f;
                dw[c][e] += d[c][e] * v[c][e];
                db[c][e] += d[c][e];
                d[c][e] *= w[c][e];
                sa += d[c][e];
                sax += d[c][e] * v[c][e];
            }
        if (!dx.p) continue;
        const float ma = sum(sa) * inv, max = sum(sax) * inv;
        if (!live) continue;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * L + lane) * VEC;
            float out[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) out[e] = rstd * (d[c][e] - ma - v[c][e] * max);
            store_pack<T, VEC>(dx.p + particle * dx.particle + r * dx.row + col, s.width - col, out);
        }
    }
    if (!partials) return;
    float *const mine = partials + (int64_t)blockIdx.x * 2 * s.width;
    if constexpr (kTeams<L> == 1) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * L + lane) * VEC;
            store_pack<float, VEC>(mine + col, s.width - col, dw[c]);
            store_pack<float, VEC>(mine + s.width + col, s.width - col, db[c]);
        }
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                sums[(c * VEC + e) * kTeamBlock<L> + threadIdx.x] = dw[c][e];
                sums[(E + c * VEC + e) * kTeamBlock<L> + threadIdx.x] = db[c][e];
            }
        __syncthreads();
        for (int k = threadIdx.x; k < 2 * E * L; k += kTeamBlock<L>) {
            const int which = k / (E * L), e = k / L % E, l = k % L;
            float total = 0.f;
#pragma unroll
            for (int t = 0; t < kTeams<L>; ++t) total += sums[(which * E + e) * kTeamBlock<L> + t * L + l];
            const int col = (e / VEC * L + l) * VEC + e % VEC;
            if (col < s.width) mine[which * s.width + col] = total;
        }
    }
}

// Sums of a particle's partials, in the same order every time: 64 columns per workgroup, its sixteen waves take every
// sixteenth partial, four of them in flight, and their sums are added in order.
constexpr int kReduceWaves = 16;
static __global__ __launch_bounds__(64 * kReduceWaves) void norm_reduce_kernel(const float *partials, int blocks, int width, int column_groups, Params dweight,
                                                                        Params dbias, bool accumulate)
{
    __shared__ double sums[kReduceWaves][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t particle = blockIdx.x / column_groups;
    const int col = (blockIdx.x % column_groups) * 64 + lane; // of 2 * width
    double total = 0.0;
    if (col < 2 * width) {
        const float *const p = partials + particle * blocks * 2 * (int64_t)width + col;
        int b = wave;
        for (; b + 3 * kReduceWaves < blocks; b += 4 * kReduceWaves) {
            float v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = p[(int64_t)(b + k * kReduceWaves) * 2 * width];
#pragma unroll
            for (int k = 0; k < 4; ++k) total += (double)v[k];
        }
        for (; b < blocks; b += kReduceWaves) total += (double)p[(int64_t)b * 2 * width];
    }
    sums[wave][lane] = total;
    __syncthreads();
    if (wave != 0 || col >= 2 * width) return;
    const Params &out = col < width ? dweight : dbias;
    if (!out.p) return;
    float *const p = const_cast<float *>(out.p) + particle * out.stride + (col < width ? col : col - width);
    double v = 0.0;
#pragma unroll
    for (int w = 0; w < kReduceWaves; ++w) v += sums[w][lane];
    *p = (float)(accumulate ? v + (double)*p : v);
}

} // namespace svgd
