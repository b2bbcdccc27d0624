// The products of a gated feed-forward block and of its backward pass, for all particles in one launch each:
//     g = x Wg^T, u = x Wu^T, h = act(g) u                       gate_up_kernel   (the activation in its epilogue)
//     y = h Wd^T                                                 down_kernel
//     dh = dy Wd, dg = dh u act'(g), du = dh act(g)              hidden_grad_kernel (these in its epilogue)
//     dx = dg Wg + du Wu                                         input_grad_kernel
//     dWg = dg^T x, dWu = du^T x, dWd = dy^T h                   weight_grad_kernel
//
// All of them are one tile product, C[j][i] = sum_k A[i][k] B[j][k], 128 x 128 values of C per workgroup of four waves
// of 64 x 64.  Operands are fp32 or 16 bits wide in memory; on their way into LDS they become bf16 parts whose sum is the value
// EXACTLY (split3: three parts of an fp32 value, two of an fp16 one, one of a bf16 one), and the matrix cores
// add up the products of parts that are not below 2^-24 of the whole: six for two fp32 operands, three for fp32 and bf16.  That is
// the accuracy of fp32 products at 2.5 PFLOP/s / 6 (or / 3), where the fp32 matrix instructions end at 157 TFLOP/s; and
// since each part is read from LDS once for several products, LDS keeps up with half the traffic a
// plain bf16 product needs.
#pragma once
#include "layer_common.hpp"

namespace svgd {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kTile = 128;  // rows of A and of B per workgroup
constexpr int kTileK = 32;  // columns of both per step

template <class T> constexpr int kParts = 3;
template <> constexpr int kParts<f16_t> = 2;
template <> constexpr int kParts<bf16_t> = 1;

// An operand's tile in LDS: one plane per part, each kTile rows of four 16-byte units (8 values of k).  Two rows share 128
// bytes; which half a row takes and where its units lie in it is permuted so that neither 8 rows in succession nor 8
// every-second rows (what eight lanes read or write at a time) meet in a bank.
constexpr int kPlane = kTile * 4; // units
__device__ __forceinline__ int unit_of(int row, int kg) { return (row >> 1) * 8 + (((row ^ (row >> 3)) & 1) << 2) + (kg ^ ((row >> 1) & 3)); }

template <int P>
__device__ __forceinline__ void split_parts(f32x4 a, f32x4 b, const SplitConst &sc, bf16x8 (&out)[P])
{
    if constexpr (P == 3) {
        const Split3 s = split3(a, b, sc);
        out[0] = s.h;
        out[1] = s.m;
        out[2] = s.l;
    } else {
        static_assert(P == 2, "one part is a copy");
        const bf16x2 neg_lo = __builtin_bit_cast(bf16x2, sc.neg_lo), neg_hi = __builtin_bit_cast(bf16x2, sc.neg_hi);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f32x2 v = k < 2 ? f32x2{a[2 * k], a[2 * k + 1]} : f32x2{b[2 * k - 4], b[2 * k - 3]};
            const bf16x2 h = __builtin_convertvector(v, bf16x2);
            v = f32x2{__builtin_amdgcn_fdot2_f32_bf16(h, neg_lo, v[0], false), __builtin_amdgcn_fdot2_f32_bf16(h, neg_hi, v[1], false)};
            const bf16x2 m = __builtin_convertvector(v, bf16x2);
            out[0][2 * k] = h[0];
            out[0][2 * k + 1] = h[1];
            out[1][2 * k] = m[0];
            out[1][2 * k + 1] = m[1];
        }
    }
}

// Eight values of one row, as P parts.
template <class T, int P>
__device__ __forceinline__ void to_parts(const T (&v)[8], const SplitConst &sc, bf16x8 (&out)[P])
{
    if constexpr (P == 1) {
        static_assert(sizeof(T) == 2, "bf16 values");
#pragma unroll
        for (int e = 0; e < 8; ++e) out[0][e] = v[e];
    } else {
        split_parts<P>(f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]}, f32x4{(float)v[4], (float)v[5], (float)v[6], (float)v[7]}, sc, out);
    }
}

// An operand whose k is contiguous in memory: each thread brings 8 values of k of rows tid / 4 and tid / 4 + 64.
template <class T, int P> struct AlongK {
    const T *row[2];
    T v[2][8];
    template <class F> __device__ __forceinline__ AlongK(F row_start)
    {
        row[0] = row_start(threadIdx.x >> 2);
        row[1] = row_start((threadIdx.x >> 2) + 64);
    }
    // Columns k0 .. k0 + 31; those from K on count as 0 and are not read.
    __device__ __forceinline__ void fetch(int64_t k0, int64_t K)
    {
        const int64_t k = k0 + (threadIdx.x & 3) * 8;
        if (k0 + kTileK <= K) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                constexpr int W = 16 / sizeof(T);
#pragma unroll
                for (int q = 0; q < 8; q += W) {
                    const typename Pack<T, W>::raw r = *reinterpret_cast<const typename Pack<T, W>::type *>(row[t] + k + q);
#pragma unroll
                    for (int e = 0; e < W; ++e) v[t][q + e] = r[e];
                }
            }
        } else {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const T x = row[t][k + e < K ? k + e : K - 1];
                    v[t][e] = k + e < K ? x : (T)0.f;
                }
        }
    }
    __device__ __forceinline__ void store(bf16x8 *lds, const SplitConst &sc) const
    {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            bf16x8 parts[P];
            to_parts<T, P>(v[t], sc, parts);
            const int u = unit_of((threadIdx.x >> 2) + 64 * t, threadIdx.x & 3);
#pragma unroll
            for (int p = 0; p < P; ++p) lds[p * kPlane + u] = parts[p];
        }
    }
};

// An operand whose rows are contiguous in memory, k after k `stride` apart: each thread brings rows 2 l and 2 l + 1, l its
// lane, of 8 values of k, one such group per wave.  `count`: how many of the tile's rows there are.
template <class T, int P> struct AcrossK {
    const T *base;
    int64_t stride;
    int count;
    T v[2][8];
    __device__ __forceinline__ AcrossK(const T *b, int64_t s, int64_t left) : base(b), stride(s), count(left < kTile ? (int)left : kTile) {}
    __device__ __forceinline__ void fetch(int64_t k0, int64_t K)
    {
        const int r = 2 * (threadIdx.x & 63);
        const int64_t k = k0 + (threadIdx.x >> 6) * 8;
        if (k0 + kTileK <= K && count == kTile) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const typename Pack<T, 2>::raw x = *reinterpret_cast<const typename Pack<T, 2>::type *>(base + (k + e) * stride + r);
                v[0][e] = x[0];
                v[1][e] = x[1];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const T *line = base + (k + e < K ? k + e : K - 1) * stride;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const T x = line[r + t < count ? r + t : count - 1];
                    v[t][e] = k + e < K ? x : (T)0.f;
                }
            }
        }
    }
    __device__ __forceinline__ void store(bf16x8 *lds, const SplitConst &sc) const
    {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            bf16x8 parts[P];
            to_parts<T, P>(v[t], sc, parts);
            const int u = unit_of(2 * (threadIdx.x & 63) + t, threadIdx.x >> 6);
#pragma unroll
            for (int p = 0; p < P; ++p) lds[p * kPlane + u] = parts[p];
        }
    }
};

// The wave's 64 x 64 values of C: block (ib, jb) of 32 x 32, in it value r of a lane is
// i = 8 (r / 4) + 4 (lane / 32) + r % 4, j = lane % 32.
struct Acc {
    f32x16 c[2][2];
    __device__ __forceinline__ Acc()
    {
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b) c[a][b] = f32x16{};
    }
};

// Adds the product over K columns to acc.  Products of parts pa, pb with pa + pb beyond the last part are below 2^-24
// (three parts; 2^-16 with two) of the whole and left out.
template <int PA, int PB, class LA, class LB>
__device__ __forceinline__ void tile_product(LA &a, LB &b, int64_t K, Acc &acc, bf16x8 *lds)
{
    constexpr int kOrder = (PA > PB ? PA : PB) - 1;
    const SplitConst sc = split_const();
    bf16x8 *const lds_b = lds + PA * kPlane;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wi = wave & 1, wj = wave >> 1;
    const int frag[2] = {unit_of(lane & 31, lane >> 5), unit_of(lane & 31, 2 + (lane >> 5))};
    if (K > 0) {
        a.fetch(0, K);
        b.fetch(0, K);
    }
    for (int64_t k0 = 0; k0 < K; k0 += kTileK) {
        __syncthreads(); // the step before has been read
        a.store(lds, sc);
        b.store(lds_b, sc);
        __syncthreads();
        if (k0 + kTileK < K) {
            a.fetch(k0 + kTileK, K);
            b.fetch(k0 + kTileK, K);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            bf16x8 fa[2][PA], fb[2][PB];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
#pragma unroll
                for (int p = 0; p < PA; ++p) fa[q][p] = lds[p * kPlane + (wi * 64 + q * 32) * 4 + frag[s]];
#pragma unroll
                for (int p = 0; p < PB; ++p) fb[q][p] = lds_b[p * kPlane + (wj * 64 + q * 32) * 4 + frag[s]];
            }
#pragma unroll
            for (int pa = 0; pa < PA; ++pa)
#pragma unroll
                for (int pb = 0; pb < PB; ++pb)
                    if (pa + pb <= kOrder) {
#pragma unroll
                        for (int ib = 0; ib < 2; ++ib)
#pragma unroll
                            for (int jb = 0; jb < 2; ++jb)
                                acc.c[ib][jb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[ib][pa], fb[jb][pb], acc.c[ib][jb], 0, 0, 0);
                    }
        }
    }
}

// Which tile a workgroup computes.  Workgroups go round the eight dies in turn: every die gets tiles that follow one another, so
// that the operands they share meet in its L2; and they follow one another in blocks of kBand tiles of j.
constexpr int kDies = 8, kBand = 8;
struct TileGrid {
    int ti, tj, per_die, total;
    __host__ TileGrid(int n, int64_t i, int64_t j) : ti((int)i), tj((int)j), per_die(0), total(0)
    {
        const int64_t t = (int64_t)n * i * j;
        total = t > (1 << 24) - kDies ? -1 : (int)t; // (more than memory holds, and than a launch takes)
        per_die = total < 0 ? 0 : (int)((t + kDies - 1) / kDies);
    }
    __host__ int blocks() const { return per_die * kDies; }
    // false: nothing to do
    __device__ __forceinline__ bool at(int &particle, int &i, int &j) const
    {
        const int id = (blockIdx.x % kDies) * per_die + blockIdx.x / kDies;
        if (id >= total) return false;
        particle = id / (ti * tj);
        const int r = id - particle * ti * tj;
        const int band = r / (ti * kBand), left = r - band * ti * kBand;
        const int high = tj - band * kBand < kBand ? tj - band * kBand : kBand;
        i = left / high;
        j = band * kBand + left - i * high;
        return true;
    }
};

template <int ACT> __device__ __forceinline__ void activate(float g, float &a, float &slope)
{
    if constexpr (ACT == SVGD_SILU) {
        const float s = 1.f / (1.f + expf(-g));
        a = g * s;
        slope = s * (1.f + g * (1.f - s));
    } else {
        const float cdf = 0.5f * (1.f + erff(g * 0.70710678118654752f));
        a = g * cdf;
        slope = cdf + g * 0.39894228040143268f * expf(-0.5f * g * g);
    }
}

struct FfnShape {
    int64_t rows, width, hidden, hidden_ld; // hidden_ld: row stride of g, u, h, dg, du in the buffers
};
template <class T> struct Rows {
    T *p;
    int64_t particle, row; // strides
};

// calls f(i, j, quad) for every four values of C that a lane holds side by side: C[j][i .. i + 3] of the tile
template <class F> __device__ __forceinline__ void each_quad(const Acc &acc, F f)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int i0 = (wave & 1) * 64 + 4 * (lane >> 5), j0 = (wave >> 1) * 64 + (lane & 31);
#pragma unroll
    for (int ib = 0; ib < 2; ++ib)
#pragma unroll
        for (int jb = 0; jb < 2; ++jb)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x16 &c = acc.c[ib][jb];
                f(i0 + ib * 32 + q * 8, j0 + jb * 32, f32x4{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]});
            }
}

// Of the tile's 128 rows of A every wave's 64 are 32 of gate and the same 32 of up, so that a lane has g and u of
// the same values.
template <class T, int ACT, bool SAVE>
__global__ __launch_bounds__(256, 2) void gate_up_kernel(FfnShape s, TileGrid grid, Rows<const T> x, Params gate, Params up, float *h, float *g_out,
                                                         float *u_out)
{
    __shared__ bf16x8 lds[(3 + kParts<T>)*kPlane];
    int particle, ti, tj;
    if (!grid.at(particle, ti, tj)) return;
    const float *const wg = gate.p + particle * gate.stride, *const wu = up.p + particle * up.stride;
    const T *const xs = x.p + particle * x.particle;
    const int64_t i0 = (int64_t)ti * (kTile / 2), j0 = (int64_t)tj * kTile;
    AlongK<float, 3> a([&](int r) {
        int64_t i = i0 + (r >> 6) * 32 + (r & 31);
        if (i >= s.hidden) i = s.hidden - 1;
        return ((r >> 5) & 1 ? wu : wg) + i * s.width;
    });
    AlongK<T, kParts<T>> b([&](int r) { return xs + (j0 + r < s.rows ? j0 + r : s.rows - 1) * x.row; });
    Acc acc;
    tile_product<3, kParts<T>>(a, b, s.width, acc, lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t i = i0 + (wave & 1) * 32 + 4 * (lane >> 5);
#pragma unroll
    for (int jb = 0; jb < 2; ++jb) {
        const int64_t j = j0 + (wave >> 1) * 64 + jb * 32 + (lane & 31);
        if (j >= s.rows) continue;
        const int64_t at = (particle * s.rows + j) * s.hidden_ld + i;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (i + 8 * q >= s.hidden_ld) continue; // (the columns from hidden to hidden_ld are never used)
            f32x4 g, u, v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                g[e] = acc.c[0][jb][4 * q + e];
                u[e] = acc.c[1][jb][4 * q + e];
                float act, slope;
                activate<ACT>(g[e], act, slope);
                v[e] = act * u[e];
            }
            *reinterpret_cast<f32x4 *>(h + at + 8 * q) = v;
            if constexpr (SAVE) {
                *reinterpret_cast<f32x4 *>(g_out + at + 8 * q) = g;
                *reinterpret_cast<f32x4 *>(u_out + at + 8 * q) = u;
            }
        }
    }
}

// Two parts of each operand are enough where the result is rounded to 16 bits: what is left out is below 2^-16 of a product.
template <class T> constexpr int kHiddenParts = sizeof(T) == 4 ? 3 : 2;

template <class T>
__global__ __launch_bounds__(256, 2) void down_kernel(FfnShape s, TileGrid grid, const float *h, Params down, Rows<T> y)
{
    constexpr int P = kHiddenParts<T>;
    __shared__ bf16x8 lds[2 * P * kPlane];
    int particle, ti, tj;
    if (!grid.at(particle, ti, tj)) return;
    const float *const w = down.p + particle * down.stride, *const hs = h + particle * s.rows * s.hidden_ld;
    const int64_t i0 = (int64_t)ti * kTile, j0 = (int64_t)tj * kTile;
    AlongK<float, P> a([&](int r) { return w + (i0 + r < s.width ? i0 + r : s.width - 1) * s.hidden; });
    AlongK<float, P> b([&](int r) { return hs + (j0 + r < s.rows ? j0 + r : s.rows - 1) * s.hidden_ld; });
    Acc acc;
    tile_product<P, P>(a, b, s.hidden, acc, lds);
    each_quad(acc, [&](int i, int j, f32x4 c) {
        if (j0 + j >= s.rows || i0 + i >= s.width) return;
        const float v[4] = {c[0], c[1], c[2], c[3]};
        const int64_t left = s.width - i0 - i;
        store_pack<T, 4>(y.p + particle * y.particle + (j0 + j) * y.row + i0 + i, left < 4 ? (int)left : 4, v);
    });
}

template <class T, int ACT>
__global__ __launch_bounds__(256, 2) void hidden_grad_kernel(FfnShape s, TileGrid grid, Rows<const T> dy, Params down, const float *g, const float *u,
                                                             float *dg, float *du)
{
    __shared__ bf16x8 lds[(3 + kParts<T>)*kPlane];
    int particle, ti, tj;
    if (!grid.at(particle, ti, tj)) return;
    const int64_t i0 = (int64_t)ti * kTile, j0 = (int64_t)tj * kTile;
    const T *const dys = dy.p + particle * dy.particle;
    AcrossK<float, 3> a(down.p + particle * down.stride + i0, s.hidden, s.hidden - i0);
    AlongK<T, kParts<T>> b([&](int r) { return dys + (j0 + r < s.rows ? j0 + r : s.rows - 1) * dy.row; });
    Acc acc;
    tile_product<3, kParts<T>>(a, b, s.width, acc, lds);
    each_quad(acc, [&](int i, int j, f32x4 c) {
        if (j0 + j >= s.rows || i0 + i >= s.hidden_ld) return;
        const int64_t at = (particle * s.rows + j0 + j) * s.hidden_ld + i0 + i;
        const f32x4 gv = *reinterpret_cast<const f32x4 *>(g + at), uv = *reinterpret_cast<const f32x4 *>(u + at);
        f32x4 dgv, duv;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float act, slope;
            activate<ACT>(gv[e], act, slope);
            dgv[e] = c[e] * uv[e] * slope;
            duv[e] = c[e] * act;
        }
        *reinterpret_cast<f32x4 *>(dg + at) = dgv;
        *reinterpret_cast<f32x4 *>(du + at) = duv;
    });
}

template <class T>
__global__ __launch_bounds__(256, 2) void input_grad_kernel(FfnShape s, TileGrid grid, const float *dg, const float *du, Params gate, Params up, Rows<T> dx)
{
    constexpr int P = kHiddenParts<T>;
    __shared__ bf16x8 lds[2 * P * kPlane];
    int particle, ti, tj;
    if (!grid.at(particle, ti, tj)) return;
    const int64_t i0 = (int64_t)ti * kTile, j0 = (int64_t)tj * kTile;
    Acc acc;
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
        const float *const w = half ? up.p + particle * up.stride : gate.p + particle * gate.stride;
        const float *const d = (half ? du : dg) + particle * s.rows * s.hidden_ld;
        AcrossK<float, P> a(w + i0, s.width, s.width - i0);
        AlongK<float, P> b([&](int r) { return d + (j0 + r < s.rows ? j0 + r : s.rows - 1) * s.hidden_ld; });
        tile_product<P, P>(a, b, s.hidden, acc, lds);
    }
    each_quad(acc, [&](int i, int j, f32x4 c) {
        if (j0 + j >= s.rows || i0 + i >= s.width) return;
        const float v[4] = {c[0], c[1], c[2], c[3]};
        const int64_t left = s.width - i0 - i;
        store_pack<T, 4>(dx.p + particle * dx.particle + (j0 + j) * dx.row + i0 + i, left < 4 ? (int)left : 4, v);
    });
}

// out[j][i] (+)= sum over the rows t of b[t][j] a[t][i], `wide` values of i and `high` of j, for one or two pairs (b, out).
template <class TA, class TB>
__global__ __launch_bounds__(256, 2) void weight_grad_kernel(int64_t rows, int64_t wide, int64_t high, TileGrid grid, int tiles_high, Rows<const TA> a_rows,
                                                             Rows<const TB> b_rows0, Rows<const TB> b_rows1, Params out0, Params out1, bool accumulate)
{
    constexpr int PA = kParts<TA>, PB = kParts<TB>;
    __shared__ bf16x8 lds[(PA + PB) * kPlane];
    int particle, ti, tj;
    if (!grid.at(particle, ti, tj)) return;
    const bool second = tj >= tiles_high;
    if (second) tj -= tiles_high;
    const Rows<const TB> b_rows = second ? b_rows1 : b_rows0;
    float *const out = const_cast<float *>(second ? out1.p + particle * out1.stride : out0.p + particle * out0.stride);
    const int64_t i0 = (int64_t)ti * kTile, j0 = (int64_t)tj * kTile;
    AcrossK<TA, PA> a(a_rows.p + particle * a_rows.particle + i0, a_rows.row, wide - i0);
    AcrossK<TB, PB> b(b_rows.p + particle * b_rows.particle + j0, b_rows.row, high - j0);
    Acc acc;
    tile_product<PA, PB>(a, b, rows, acc, lds);
    each_quad(acc, [&](int i, int j, f32x4 c) {
        if (j0 + j >= high || i0 + i >= wide) return;
        float *const p = out + (j0 + j) * wide + i0 + i;
        const int64_t left = wide - i0 - i;
        float v[4] = {c[0], c[1], c[2], c[3]};
        if (accumulate) {
            float old[4];
            load_pack<float, 4>(p, left < 4 ? (int)left : 4, old);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += old[e];
        }
        store_pack<float, 4>(p, left < 4 ? (int)left : 4, v);
    });
}

} // namespace svgd
