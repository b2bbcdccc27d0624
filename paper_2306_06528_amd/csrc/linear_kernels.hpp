// Linear maps with bias, activation and residual, and their backward pass: the tile products of ffn_kernels.hpp with epilogues of their
// own.
//     z = x W^T + b, y = act(z) + residual          linear_forward_kernel, or thin_linear_kernel for few rows
//     dz = dy act'(z), db = sum dz                  linear_slope_kernel (dz only where there is an activation: otherwise it is dy)
//     dx = dz W, dW = dz^T x                        linear_gradients_kernel
// x has one, two or three parts by its type and W three, so a product has fp32's accuracy; without an activation dW of 16-bit calls is a
// product of 16-bit operands, of one part each for bf16: exact at a sixth of the cost.  The matrix cores bound the large products, reading
// the weights those of few rows. 8 x 4,096 x 1,024 x 1,024 bf16: forward 256 to 266 us (206 Gflop of bf16 products, 780 TFLOP/s: two rounds
// of tiles, whose first loads and epilogues nothing covers), gradients 256 to 269 (275, 1,050 TFLOP/s), sums of dy's columns 24 (67 MB); 5
// x 1,003 x 333 x 501 fp32 tanh: forward 35, gradients 39; 16 x 1 x 256 x 768 fp32: 5.0.
#pragma once
#include "ffn_thin_kernels.hpp"
#include "linear_rules.hpp"
#include "../../include/svgd_attention.h"

namespace svgd {

// act(z) and act'(z); `kind` is the same for all threads
__device__ __forceinline__ void activate(int kind, float z, float &a, float &slope)
{
    if (kind == SVGD_SILU) {
        activate<SVGD_SILU>(z, a, slope);
    } else if (kind == SVGD_GELU) {
        activate<SVGD_GELU>(z, a, slope);
    } else if (kind == SVGD_TANH) {
        a = tanhf(z);
        const float e = expf(-2.f * fabsf(z)); // 1 - tanh^2 = 4 e / (1 + e)^2, which keeps its digits where tanh is near 1
        slope = 4.f * e / ((1.f + e) * (1.f + e));
    } else if (kind == SVGD_RELU) {
        a = z > 0.f ? z : z == z ? 0.f : z;
        slope = z > 0.f ? 1.f : z == z ? 0.f : z;
    } else {
        a = z;
        slope = 1.f;
    }
}

struct LinearShape {
    int n, activation;
    int64_t rows, width, out, out_ld, width_ld;
};

// What becomes of z once it is summed up.
template <class T> struct LinearEnd {
    const float *bias; // of the particle, or null
    const T *residual; // of the particle, or null
    int64_t residual_row;
    T *y; // of the particle
    int64_t y_row;
    float *z; // of the particle, or null
    int64_t z_row;
    // values i .. i + 3 of row j, those from `out` on not there
    __device__ __forceinline__ void operator()(const LinearShape &s, int64_t i, int64_t j, f32x4 c) const
    {
        const int64_t left = s.out - i;
        if (bias) {
            float b[4];
            load_pack<float, 4>(bias + i, left < 4 ? (int)left : 4, b);
#pragma unroll
            for (int e = 0; e < 4; ++e) c[e] += b[e];
        }
        if (z) *reinterpret_cast<f32x4 *>(z + j * z_row + i) = c; // (what is beyond `out` is not used)
        if (s.activation != SVGD_NO_ACTIVATION) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float a, slope;
                activate(s.activation, c[e], a, slope);
                c[e] = a;
            }
        }
        if (residual) {
            float r[4];
            load_pack<T, 4>(residual + j * residual_row + i, left < 4 ? (int)left : 4, r);
#pragma unroll
            for (int e = 0; e < 4; ++e) c[e] += r[e];
        }
        store_quad(y + j * y_row + i, c, 0, left);
    }
};
template <class T> struct LinearOut {
    Params bias;
    Rows<const T> residual;
    Rows<T> y;
    float *z;
    __device__ __forceinline__ LinearEnd<T> of(const LinearShape &s, int particle) const
    {
        return {bias.p ? bias.p + particle * bias.stride : nullptr, residual.p ? residual.p + particle * residual.particle : nullptr, residual.row,
                y.p + particle * y.particle, y.row, z ? z + particle * s.rows * s.out_ld : nullptr, s.out_ld};
    }
};

// partial: with more than one part, their sums [part][particle][row][out_ld]
template <class TL, class T>
SVGD_TILE_KERNEL void linear_forward_kernel(LinearShape s, TileGrid grid, Rows<const T> x, Params weight, LinearOut<T> to, float *partial)
{
    constexpr int P = kParts<T>;
    __shared__ bf16x8 lds[2 * P * TL::kPlane];
    __shared__ float scratches[TL::kWaves][kScratch];
    float *const scratch = scratches[wave_of_block()];
    int particle, part, ti, tj;
    if (!grid.at(blockIdx.x, particle, part, ti, tj)) return;
    const float *const w = weight.p + particle * weight.stride;
    const int64_t i0 = (int64_t)ti * TL::kI, j0 = (int64_t)tj * TL::kJ, iw = i0 + wave_of_block() * 64;
    const int64_t first = iw < s.out ? iw : s.out - 1;
    RowsOfA<3, 1> a(w + first * s.width, w, s.out - first, s.width);
    RowsOfB<TL, T, P> b(x.p + particle * x.particle + j0 * x.row, x.row, s.rows - j0);
    Acc<TL::kBlocksJ> acc;
    tile_product<TL, 3, P, true>(a, b, grid.begin(part), grid.end(part), acc, lds, scratch);
    const LinearEnd<T> end = to.of(s, particle);
    float *const sums = partial + ((int64_t)part * s.n + particle) * s.rows * s.out_ld;
    each_quad<TL, false>(acc, iw, s.out, j0, scratch, [&](int64_t i, int64_t j, f32x4 c, int64_t) {
        if (j >= s.rows) return;
        if (grid.splits > 1) *reinterpret_cast<f32x4 *>(sums + j * s.out_ld + i) = c;
        else end(s, i, j, c);
    });
}

// The parts' sums, in order, and what becomes of them.
template <class T> __global__ __launch_bounds__(256) void linear_join_kernel(LinearShape s, const float *partial, int parts, LinearOut<T> to)
{
    const int64_t quads = s.out_ld / 4, k = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (k >= s.n * s.rows * quads) return;
    const int64_t line = k / quads, i = (k - line * quads) * 4, particle = line / s.rows, j = line - particle * s.rows;
    const int64_t each = s.n * s.rows * s.out_ld;
    const float *p = partial + line * s.out_ld + i;
    f32x4 total = {0.f, 0.f, 0.f, 0.f};
    for (int part = 0; part < parts; ++part) total += *reinterpret_cast<const f32x4 *>(p + part * each);
    to.of(s, (int)particle)(s, i, j, total);
}

// Up to 16 JB rows: every weight is read once, by a wave of its own (ffn_thin_kernels.hpp).
template <class T, int JB> SVGD_THIN_KERNEL void thin_linear_kernel(LinearShape s, ThinGrid grid, Rows<const T> x, Params weight, LinearOut<T> to)
{
    constexpr int P = kParts<T>, U = JB == 1 ? 2 : 4 / JB, kPart = kThinPart<JB, 2>;
    __shared__ f32x4 parts[kThinWaves * kPart];
    f32x4 *const slots = parts + wave_of_block() * kPart;
    const int particle = grid.particle();
    const int64_t i0 = grid.first();
    const ThinRows<float>::From w(weight.p + particle * weight.stride + i0 * s.width, s.width, s.out - 1 - i0);
    const ThinFrom<T, JB> xr(x.p + particle * x.particle, x.row, s.rows);
    const SplitConst sc = split_const();
    ThinRows<float> a[U];
    ThinRows<T> r[U][JB];
    f32x4 c[JB];
#pragma unroll
    for (int b = 0; b < JB; ++b) c[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    thin_steps<U>(
        s.width,
        [&](int q, int64_t k) {
            a[q].load(w, k);
#pragma unroll
            for (int b = 0; b < JB; ++b) r[q][b].load(xr.of[b], k);
        },
        [&](int64_t k) {
            a[0].load_last(w, k, s.width);
#pragma unroll
            for (int b = 0; b < JB; ++b) r[0][b].load_last(xr.of[b], k, s.width);
        },
        [&](int q) {
            wave_sync();
            a[q].stage(slots);
            r[q][0].stage(slots + kSlot);
            wave_sync();
            bf16x8 ap[3];
            thin_parts<float, 3>(slots, sc, ap);
            each_thin_row<T, JB>(r[q], slots + kSlot, sc, [&](int b, const bf16x8(&xp)[P]) { thin_product<3, P>(ap, xp, c[b]); });
        });
    const LinearEnd<T> end = to.of(s, particle);
    join_waves<JB, 1>(c, parts, kPart, [&](int b, int ii, int jj, const float (&v)[1]) {
        const int64_t j = b * 16 + jj, i = i0 + ii;
        if (j >= s.rows || i >= s.out) return;
        float z = v[0], y, slope;
        if (end.bias) z += end.bias[i];
        if (end.z) end.z[j * end.z_row + i] = z;
        activate(s.activation, z, y, slope);
        if (end.residual) y += (float)end.residual[j * end.residual_row + i];
        end.y[j * end.y_row + i] = (T)y;
    });
}

// dz (null: not wanted) of some rows, and the sums of their columns (null: not wanted) to sums[part][particle][out], or where there is one
// part to the bias's gradient: 64 lanes have four columns each, the four waves every fourth row.
template <class T, bool ACT>
__global__ __launch_bounds__(256) void linear_slope_kernel(LinearShape s, int64_t per, int parts, int groups, Rows<const T> dy, const float *z, float *dz, float *sums, Params dbias,
                                                           bool accumulate)
{
    __shared__ f32x4 waves[4][64];
    int id = blockIdx.x;
    const int group = id % groups;
    id /= groups;
    const int part = id % parts, particle = id / parts;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t i = (int64_t)group * 256 + 4 * lane, last = (part + 1) * per < s.rows ? (part + 1) * per : s.rows;
    const int left = s.out - i < 4 ? (int)(s.out - i) : 4;
    f32x4 total = {0.f, 0.f, 0.f, 0.f};
    if (left > 0) {
        constexpr int U = ACT ? 2 : 8;
#pragma unroll U
        for (int64_t j = part * per + wave; j < last; j += 4) {
            float g[4];
            load_pack<T, 4>(dy.p + particle * dy.particle + j * dy.row + i, left, g);
            if constexpr (ACT) {
                const int64_t at = (particle * s.rows + j) * s.out_ld + i;
                const f32x4 zv = *reinterpret_cast<const f32x4 *>(z + at);
                f32x4 d;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float a, slope;
                    activate(s.activation, zv[e], a, slope);
                    d[e] = e < left ? g[e] * slope : 0.f;
                    g[e] = d[e];
                }
                if (dz) *reinterpret_cast<f32x4 *>(dz + at) = d;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) total[e] += g[e];
        }
    }
    if (!dbias.p) return;
    waves[wave][lane] = total;
    __syncthreads();
    if (wave != 0 || left <= 0) return;
    total = (waves[0][lane] + waves[1][lane]) + (waves[2][lane] + waves[3][lane]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (e >= left) continue;
        if (parts > 1) {
            sums[((int64_t)part * s.n + particle) * s.out + i + e] = total[e];
        } else {
            float *const p = const_cast<float *>(dbias.p) + particle * dbias.stride + i + e;
            *p = accumulate ? total[e] + *p : total[e];
        }
    }
}

// Parts' sums of a parameter's gradient, [part][particle][size].
struct PartSums {
    const float *partial;
    int parts; // 0: the sum is 0
    int64_t size;
    Params out; // null: none
    __host__ __device__ int64_t blocks() const { return out.p ? (size + 255) / 256 : 0; }
};

// Adds them up, in order, those of the weight and of the bias in one launch: a workgroup has 256 values of a particle.  (8 x 1,024 x 1,024
// in two parts and 1,024 in 32: 29 us, 5 x 333 x 501 in two and 501 in 62: 7.0; in a launch for each, with the particle divided out in 64
// bits, 31 + 5.2 and 5.2 + 5.3.)
static __global__ __launch_bounds__(256) void linear_sums_kernel(PartSums weight, PartSums bias, bool accumulate)
{
    const bool second = blockIdx.x >= weight.blocks();
    const int64_t size = second ? bias.size : weight.size, k = (blockIdx.x - (second ? weight.blocks() : 0)) * 256 + threadIdx.x, step = gridDim.y * size;
    const float *const partial = (second ? bias.partial : weight.partial) + blockIdx.y * size;
    float *const to = const_cast<float *>(second ? bias.out.p : weight.out.p) + blockIdx.y * (second ? bias.out.stride : weight.out.stride);
    const int parts = second ? bias.parts : weight.parts;
    if (k >= size) return;
    float total = 0.f;
#pragma unroll 8
    for (int part = 0; part < parts; ++part) total += partial[part * step + k];
    to[k] = accumulate ? total + to[k] : total;
}

// dz, of T or fp32 values, for both products.
template <class TL, class T, class TD>
SVGD_TILE_KERNEL void linear_gradients_kernel(LinearShape s, TileGrid input, Rows<const TD> dz, Params weight, Rows<T> dx, float *dx_partial, WeightGrad<T, TD> grad, bool accumulate)
{
    constexpr int P = kParts<TD>;
    __shared__ bf16x8 lds[2 * P * TL::kPlane];
    __shared__ float scratches[TL::kWaves][kScratch];
    float *const scratch = scratches[wave_of_block()];
    const int block = blockIdx.x;
    if (block >= input.per_die * kDies) {
        weight_grad_tile<TL, false, true>(grad, block - input.per_die * kDies, accumulate, lds, scratch);
        return;
    }
    int particle, part, ti, tj;
    if (!input.at(block, particle, part, ti, tj)) return;
    const int64_t i0 = (int64_t)ti * TL::kI, j0 = (int64_t)tj * TL::kJ, iw = i0 + wave_of_block() * 64;
    ColumnsOfA<float, 3> a(weight.p + particle * weight.stride, s.width, iw, s.width);
    RowsOfB<TL, TD, P> b(dz.p + particle * dz.particle + j0 * dz.row, dz.row, s.rows - j0);
    Acc<TL::kBlocksJ> acc;
    tile_product<TL, 3, P, true>(a, b, input.begin(part), input.end(part), acc, lds, scratch);
    float *const sums = dx_partial + ((int64_t)part * s.n + particle) * s.rows * s.width_ld;
    each_quad<TL, true>(acc, iw, s.width, j0, scratch, [&](int64_t i, int64_t j, f32x4 c, int64_t first) {
        if (j >= s.rows) return;
        if (input.splits > 1) store_quad(sums + j * s.width_ld + i, c, (int)(first - i), s.width - i);
        else store_quad(dx.p + particle * dx.particle + j * dx.row + i, c, (int)(first - i), s.width - i);
    });
}

} // namespace svgd
