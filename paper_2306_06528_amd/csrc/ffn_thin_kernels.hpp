// The gated feed-forward block on a few rows per particle, single tokens among them: every weight is used for at most 16 JB rows
// and comes straight from memory into the registers that the matrix instructions read, without LDS.  What bounds these
// kernels is reading the weights.  A workgroup has 16 (or 32) values of each of the rows to compute; its waves take every
// kThinWaves-th step of 32 columns of k each, so that together they read the weights' rows in pieces of 1 KiB, and
// their sums are added in LDS in the order of the waves.  On the matrix cores a weight costs its split into parts and
// 6 / 64 of an instruction, however many of the 16 rows there are; on the vector ALU it would cost one instruction per row.
#pragma once
#include "ffn_kernels.hpp"

namespace svgd {

constexpr int kThinWaves = 8, kThinBlock = 64 * kThinWaves;
constexpr int kThinStride = kThinWaves * kTileK; // columns between two steps of a wave

// A wave's operand of 16 rows: lane l has row l % 16, columns (l / 16) * 8 + 0 .. 7 of a step.  K is contiguous: `row` is
// the start of the lane's row.
template <class T> struct ThinRow {
    T v[8];
    __device__ __forceinline__ void load(const T *row, int64_t k)
    {
        constexpr int W = 16 / sizeof(T);
#pragma unroll
        for (int q = 0; q < 8; q += W) {
            const typename Pack<T, W>::raw r = *reinterpret_cast<const typename Pack<T, W>::type *>(row + k + q);
#pragma unroll
            for (int e = 0; e < W; ++e) v[q + e] = r[e];
        }
    }
    __device__ __forceinline__ void load_last(const T *row, int64_t k, int64_t K) // columns from K on are 0 and not read
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const T x = row[k + e < K ? k + e : K - 1];
            v[e] = k + e < K ? x : (T)0.f;
        }
    }
};

// Rows contiguous, k after k `stride` apart: two operands, of the even and the odd ones of 32 rows (lane l: 2 (l % 16) and the
// next), eight bytes at a time.
struct ThinColumns {
    float v[2][8];
    __device__ __forceinline__ void load(const float *column, int64_t stride, int64_t k)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const Pack<float, 2>::raw r = *reinterpret_cast<const Pack<float, 2>::type *>(column + (k + e) * stride);
            v[0][e] = r[0];
            v[1][e] = r[1];
        }
    }
    // `second`: how far the second row is (0: there is none)
    __device__ __forceinline__ void load_last(const float *column, int64_t stride, int64_t k, int64_t K, int second)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float *p = column + (k + e < K ? k + e : K - 1) * stride;
            const float a = p[0], b = p[second];
            v[0][e] = k + e < K ? a : 0.f;
            v[1][e] = k + e < K ? b : 0.f;
        }
    }
};

template <int PA, int PB>
__device__ __forceinline__ void thin_product(const bf16x8 (&a)[PA], const bf16x8 (&b)[PB], f32x4 &c)
{
    constexpr int kOrder = (PA > PB ? PA : PB) - 1;
#pragma unroll
    for (int pa = 0; pa < PA; ++pa)
#pragma unroll
        for (int pb = 0; pb < PB; ++pb)
            if (pa + pb <= kOrder) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[pa], b[pb], c, 0, 0, 0);
}

// The waves' sums of N blocks of 16 x 16 (i, j), added up; f(block, i, j, sums[0 .. M)) for every value, where M
// neighbouring blocks belong together (M divides N).
template <int N, int M, class F> __device__ __forceinline__ void join_waves(const f32x4 (&c)[N], F f)
{
    __shared__ f32x4 sums[kThinWaves][N][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int b = 0; b < N; ++b) sums[wave][b][lane] = c[b];
    __syncthreads();
    for (int k = threadIdx.x; k < N / M * 256; k += kThinBlock) {
        const int block = k >> 8, i = k & 15, j = (k >> 4) & 15;
        float total[M];
#pragma unroll
        for (int m = 0; m < M; ++m) {
            total[m] = 0.f;
#pragma unroll
            for (int w = 0; w < kThinWaves; ++w) total[m] += sums[w][block * M + m][(i >> 2) * 16 + j][i & 3];
        }
        f(block, i, j, total);
    }
}

// Which 16 (32) values of which particle a workgroup computes.
struct ThinGrid {
    int per_particle, of;
    __host__ ThinGrid(int64_t size, int o) : per_particle((int)((size + o - 1) / o)), of(o) {}
    __device__ __forceinline__ int particle() const { return blockIdx.x / per_particle; }
    __device__ __forceinline__ int64_t first() const { return (int64_t)(blockIdx.x % per_particle) * of; }
};

// calls full(k) for the wave's whole steps, kUnroll at a time through load(u, k) and use(u), then the last one, if it is this
// wave's and not whole, through load_last(k) and use(0)
template <int U, class Load, class Last, class Use> __device__ __forceinline__ void thin_steps(int64_t K, Load load, Last load_last, Use use)
{
    const int wave = threadIdx.x >> 6;
    const int64_t whole = K / kTileK * kTileK; // columns of whole steps
    int64_t k = wave * kTileK;
    for (; k + (U - 1) * kThinStride < whole; k += U * kThinStride) {
#pragma unroll
        for (int u = 0; u < U; ++u) load(u, k + u * kThinStride);
#pragma unroll
        for (int u = 0; u < U; ++u) use(u);
    }
    for (; k < whole; k += kThinStride) {
        load(0, k);
        use(0);
    }
    if (k < K) { // (k is a multiple of a step: the wave whose next one this is)
        load_last(k);
        use(0);
    }
}

template <class T, int ACT, bool SAVE, int JB>
__global__ __launch_bounds__(kThinBlock) void thin_gate_up_kernel(FfnShape s, ThinGrid grid, Rows<const T> x, Params gate, Params up, float *h,
                                                                  float *g_out, float *u_out)
{
    constexpr int P = kParts<T>, U = JB > 2 ? 1 : 2;
    const int lane = threadIdx.x & 63, particle = grid.particle();
    const int64_t i0 = grid.first(), i = i0 + (lane & 15) < s.hidden ? i0 + (lane & 15) : s.hidden - 1;
    const int kl = (lane >> 4) * 8;
    const float *const wg = gate.p + particle * gate.stride + i * s.width + kl, *const wu = up.p + particle * up.stride + i * s.width + kl;
    const T *xr[JB];
#pragma unroll
    for (int b = 0; b < JB; ++b) {
        const int64_t j = b * 16 + (lane & 15);
        xr[b] = x.p + particle * x.particle + (j < s.rows ? j : s.rows - 1) * x.row + kl;
    }
    const SplitConst sc = split_const();
    ThinRow<float> g[U], u[U];
    ThinRow<T> r[U][JB];
    f32x4 c[2 * JB];
#pragma unroll
    for (int b = 0; b < 2 * JB; ++b) c[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    thin_steps<U>(
        s.width,
        [&](int q, int64_t k) {
            g[q].load(wg, k);
            u[q].load(wu, k);
#pragma unroll
            for (int b = 0; b < JB; ++b) r[q][b].load(xr[b], k);
        },
        [&](int64_t k) {
            g[0].load_last(wg, k, s.width - kl);
            u[0].load_last(wu, k, s.width - kl);
#pragma unroll
            for (int b = 0; b < JB; ++b) r[0][b].load_last(xr[b], k, s.width - kl);
        },
        [&](int q) {
            bf16x8 gp[3], up_[3], xp[P];
            to_parts<float, 3>(g[q].v, sc, gp);
            to_parts<float, 3>(u[q].v, sc, up_);
#pragma unroll
            for (int b = 0; b < JB; ++b) {
                to_parts<T, P>(r[q][b].v, sc, xp);
                thin_product<3, P>(gp, xp, c[2 * b]);
                thin_product<3, P>(up_, xp, c[2 * b + 1]);
            }
        });
    join_waves<2 * JB, 2>(c, [&](int b, int ii, int jj, const float (&v)[2]) {
        const int64_t j = b * 16 + jj;
        if (j >= s.rows || i0 + ii >= s.hidden) return;
        const int64_t at = (particle * s.rows + j) * s.hidden_ld + i0 + ii;
        float act, slope;
        activate<ACT>(v[0], act, slope);
        h[at] = act * v[1];
        if constexpr (SAVE) {
            g_out[at] = v[0];
            u_out[at] = v[1];
        }
    });
}

template <class T, int JB> __global__ __launch_bounds__(kThinBlock) void thin_down_kernel(FfnShape s, ThinGrid grid, const float *h, Params down, Rows<T> y)
{
    constexpr int U = 4 / JB;
    const int lane = threadIdx.x & 63, particle = grid.particle();
    const int64_t i0 = grid.first(), i = i0 + (lane & 15) < s.width ? i0 + (lane & 15) : s.width - 1;
    const int kl = (lane >> 4) * 8;
    const float *const w = down.p + particle * down.stride + i * s.hidden + kl;
    const float *hr[JB];
#pragma unroll
    for (int b = 0; b < JB; ++b) {
        const int64_t j = b * 16 + (lane & 15);
        hr[b] = h + (particle * s.rows + (j < s.rows ? j : s.rows - 1)) * s.hidden_ld + kl;
    }
    const SplitConst sc = split_const();
    ThinRow<float> a[U], r[U][JB];
    f32x4 c[JB];
#pragma unroll
    for (int b = 0; b < JB; ++b) c[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    thin_steps<U>(
        s.hidden,
        [&](int q, int64_t k) {
            a[q].load(w, k);
#pragma unroll
            for (int b = 0; b < JB; ++b) r[q][b].load(hr[b], k);
        },
        [&](int64_t k) {
            a[0].load_last(w, k, s.hidden - kl);
#pragma unroll
            for (int b = 0; b < JB; ++b) r[0][b].load_last(hr[b], k, s.hidden - kl);
        },
        [&](int q) {
            bf16x8 ap[3], hp[3];
            to_parts<float, 3>(a[q].v, sc, ap);
#pragma unroll
            for (int b = 0; b < JB; ++b) {
                to_parts<float, 3>(r[q][b].v, sc, hp);
                thin_product<3, 3>(ap, hp, c[b]);
            }
        });
    join_waves<JB, 1>(c, [&](int b, int ii, int jj, const float (&v)[1]) {
        const int64_t j = b * 16 + jj;
        if (j < s.rows && i0 + ii < s.width) y.p[particle * y.particle + j * y.row + i0 + ii] = (T)v[0];
    });
}

template <class T, int ACT, int JB>
__global__ __launch_bounds__(kThinBlock) void thin_hidden_grad_kernel(FfnShape s, ThinGrid grid, Rows<const T> dy, Params down, const float *g,
                                                                      const float *u, float *dg, float *du)
{
    constexpr int P = kParts<T>, U = 2;
    const int lane = threadIdx.x & 63, particle = grid.particle();
    const int64_t i0 = grid.first();
    const bool inside = i0 + 32 <= s.hidden;
    const int64_t i = i0 + 2 * (lane & 15) < s.hidden ? i0 + 2 * (lane & 15) : s.hidden - 1;
    const int second = i + 1 < s.hidden ? 1 : 0, kl = (lane >> 4) * 8;
    const float *const w = down.p + particle * down.stride + i;
    const T *dr[JB];
#pragma unroll
    for (int b = 0; b < JB; ++b) {
        const int64_t j = b * 16 + (lane & 15);
        dr[b] = dy.p + particle * dy.particle + (j < s.rows ? j : s.rows - 1) * dy.row + kl;
    }
    const SplitConst sc = split_const();
    ThinColumns a[U];
    ThinRow<T> r[U][JB];
    f32x4 c[2 * JB];
#pragma unroll
    for (int b = 0; b < 2 * JB; ++b) c[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    thin_steps<U>(
        s.width,
        [&](int q, int64_t k) {
            if (inside) a[q].load(w, s.hidden, k + kl);
            else a[q].load_last(w, s.hidden, k + kl, s.width, second);
#pragma unroll
            for (int b = 0; b < JB; ++b) r[q][b].load(dr[b], k);
        },
        [&](int64_t k) {
            a[0].load_last(w, s.hidden, k + kl, s.width, second);
#pragma unroll
            for (int b = 0; b < JB; ++b) r[0][b].load_last(dr[b], k, s.width - kl);
        },
        [&](int q) {
            bf16x8 even[3], odd[3], xp[P];
            to_parts<float, 3>(a[q].v[0], sc, even);
            to_parts<float, 3>(a[q].v[1], sc, odd);
#pragma unroll
            for (int b = 0; b < JB; ++b) {
                to_parts<T, P>(r[q][b].v, sc, xp);
                thin_product<3, P>(even, xp, c[2 * b]);
                thin_product<3, P>(odd, xp, c[2 * b + 1]);
            }
        });
    join_waves<2 * JB, 1>(c, [&](int b, int ii, int jj, const float (&v)[1]) {
        const int64_t j = (b >> 1) * 16 + jj, col = i0 + 2 * ii + (b & 1);
        if (j >= s.rows || col >= s.hidden) return;
        const int64_t at = (particle * s.rows + j) * s.hidden_ld + col;
        float act, slope;
        activate<ACT>(g[at], act, slope);
        dg[at] = v[0] * u[at] * slope;
        du[at] = v[0] * act;
    });
}

template <class T, int JB>
__global__ __launch_bounds__(kThinBlock) void thin_input_grad_kernel(FfnShape s, ThinGrid grid, const float *dg, const float *du, Params gate, Params up,
                                                                     Rows<T> dx)
{
    constexpr int U = 2;
    const int lane = threadIdx.x & 63, particle = grid.particle();
    const int64_t i0 = grid.first();
    const bool inside = i0 + 32 <= s.width;
    const int64_t i = i0 + 2 * (lane & 15) < s.width ? i0 + 2 * (lane & 15) : s.width - 1;
    const int second = i + 1 < s.width ? 1 : 0, kl = (lane >> 4) * 8;
    const SplitConst sc = split_const();
    f32x4 c[2 * JB];
#pragma unroll
    for (int b = 0; b < 2 * JB; ++b) c[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
        const float *const w = (half ? up.p + particle * up.stride : gate.p + particle * gate.stride) + i;
        const float *dr[JB];
#pragma unroll
        for (int b = 0; b < JB; ++b) {
            const int64_t j = b * 16 + (lane & 15);
            dr[b] = (half ? du : dg) + (particle * s.rows + (j < s.rows ? j : s.rows - 1)) * s.hidden_ld + kl;
        }
        ThinColumns a[U];
        ThinRow<float> r[U][JB];
        thin_steps<U>(
            s.hidden,
            [&](int q, int64_t k) {
                if (inside) a[q].load(w, s.width, k + kl);
                else a[q].load_last(w, s.width, k + kl, s.hidden, second);
#pragma unroll
                for (int b = 0; b < JB; ++b) r[q][b].load(dr[b], k);
            },
            [&](int64_t k) {
                a[0].load_last(w, s.width, k + kl, s.hidden, second);
#pragma unroll
                for (int b = 0; b < JB; ++b) r[0][b].load_last(dr[b], k, s.hidden - kl);
            },
            [&](int q) {
                bf16x8 even[3], odd[3], dp[3];
                to_parts<float, 3>(a[q].v[0], sc, even);
                to_parts<float, 3>(a[q].v[1], sc, odd);
#pragma unroll
                for (int b = 0; b < JB; ++b) {
                    to_parts<float, 3>(r[q][b].v, sc, dp);
                    thin_product<3, 3>(even, dp, c[2 * b]);
                    thin_product<3, 3>(odd, dp, c[2 * b + 1]);
                }
            });
    }
    join_waves<2 * JB, 1>(c, [&](int b, int ii, int jj, const float (&v)[1]) {
        const int64_t j = (b >> 1) * 16 + jj, col = i0 + 2 * ii + (b & 1);
        if (j < s.rows && col < s.width) dx.p[particle * dx.particle + j * dx.row + col] = (T)v[0];
    });
}

} // namespace svgd
