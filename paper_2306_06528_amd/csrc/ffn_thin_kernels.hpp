// The gated feed-forward block on a few rows per particle, single tokens among them: every weight is used for at most 16 JB rows and is
// read once, and no wave waits for another before its sums are joined.  What bounds these kernels is reading the weights.  A workgroup has
// 16 (or 32) values of each of the rows to compute; its waves take every kThinWaves-th step of 32 columns of k each, so that
// together they read the weights' rows in pieces of 1 KiB, and their sums are added in LDS in the order of the waves.  On the
// matrix cores a weight costs its split into parts and 6 / 64 of an instruction, however many of the 16 rows there are;
// on the vector ALU it would cost one instruction per row.
#pragma once
#include "ffn_kernels.hpp"

#include <utility>

namespace svgd {

constexpr int kThinWaves = 8, kThinBlock = 64 * kThinWaves;
constexpr int kThinStride = kThinWaves * kTileK; // columns between two steps of a wave

// A wave's operand of 16 rows and 32 columns, K contiguous in memory.  The matrix instructions want lane l to have row l % 16, columns
// 8 (l / 16) .. + 7, but the vector memory unit joins what 16 lanes in a row read: loaded like that, every load costs 64 accesses, which
// bound these kernels (8 x 32 rows, 1,024 x 2,730 bf16, forward: 74 us, like this 64; 1 x 64 rows fp32 39 and 30).  So eight lanes (four of 16-bit values) read 16 bytes each side by
// side, and the values change lanes in the wave's own part of LDS, as they are.
template <class T> struct ThinRows {
    static constexpr int W = 16 / sizeof(T), kPieces = kTileK / W, kAtATime = 64 / kPieces, N = 16 / kAtATime;
    typedef typename Pack<T, W>::raw raw;
    raw v[N];
    struct From {
        const T *row[N]; // the lane's piece of its rows
        // `first`: row 0; rows beyond `last`: that one again
        __device__ __forceinline__ From(const T *first, int64_t stride, int64_t last)
        {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int r = row_of(n);
                row[n] = first + (r < last ? r : last) * stride + column();
            }
        }
    };
    static __device__ __forceinline__ int row_of(int n) { return kAtATime * n + (threadIdx.x & 63) / kPieces; }
    static __device__ __forceinline__ int column() { return threadIdx.x % kPieces * W; }
    static __device__ __forceinline__ int place(int row, int piece) { return row * kPieces + (piece ^ (N == 2 ? row & 7 : (row >> 1) & 3)); } // in 16 bytes
    __device__ __forceinline__ void load(const From &from, int64_t k)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = *reinterpret_cast<const typename Pack<T, W>::type *>(from.row[n] + k);
    }
    __device__ __forceinline__ void load_last(const From &from, int64_t k, int64_t K) // columns from K on are 0 and not read
    {
        const int left = (int)(K - k) - column(); // (may be less than 1)
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const T x = from.row[n][k + (e < left ? e : left - 1)];
                v[n][e] = e < left ? x : (T)0.f;
            }
    }
    __device__ __forceinline__ void stage(f32x4 *slot) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) reinterpret_cast<raw *>(slot)[place(row_of(n), threadIdx.x % kPieces)] = v[n];
    }
    static __device__ __forceinline__ void read(const f32x4 *slot, T (&out)[8])
    {
        const int row = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const raw r = reinterpret_cast<const raw *>(slot)[place(row, N * g + q)];
#pragma unroll
            for (int e = 0; e < W; ++e) out[q * W + e] = r[e];
        }
    }
};
constexpr int kSlot = 16 * kTileK / 4; // one operand, in 16 bytes

// Forward with up to 16 rows three workgroups fit a CU, which the compiler has to be told, if a wave has one step of gate and up on its way, or two
// of down (whether the grid has so many is not looked at): 16 x 1 rows, 256 x 683 fp32 9.8 us; two workgroups and twice the steps 10.9 (8 x 5 rows, 1,024 x 2,731 bf16 55 both, 1 x 8 rows, 4,096 x
// 11,008 110 and 106).
#define SVGD_THIN_KERNEL __global__ __launch_bounds__(kThinBlock) __attribute__((amdgpu_waves_per_eu(JB == 1 ? 6 : 2)))

// A wave's part of LDS: `slots` operands, and later its sums of N blocks of 16 x 16.
template <int N, int SLOTS> constexpr int kThinPart = 64 * N > SLOTS * kSlot ? 64 * N : SLOTS * kSlot;

// The same, loaded as the matrix instructions want it, `row` being the start of the lane's row and columns: where the weights lie k after k,
// 16 lanes in a row read 128 bytes of them anyway and the detour of the activations costs more than it saves (dx of 16 x 1 rows, 256 x 683 fp32
// 15.0 us, with the detour 17.5; of 1 x 1 rows, 1,024 x 2,730 31 and 36).
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
// neighbouring blocks belong together (M divides N).  parts: LDS, `part` from one wave's to the next one's, each free for that wave to write.
template <int N, int M, class F> __device__ __forceinline__ void join_waves(const f32x4 (&c)[N], f32x4 *parts, int part, F f)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    wave_sync();
#pragma unroll
    for (int b = 0; b < N; ++b) parts[wave * part + b * 64 + lane] = c[b];
    __syncthreads();
    for (int k = threadIdx.x; k < N / M * 256; k += kThinBlock) {
        const int block = k >> 8, i = k & 15, j = (k >> 4) & 15;
        float total[M];
#pragma unroll
        for (int m = 0; m < M; ++m) {
            total[m] = 0.f;
#pragma unroll
            for (int w = 0; w < kThinWaves; ++w) total[m] += parts[w * part + (block * M + m) * 64 + (i >> 2) * 16 + j][i & 3];
        }
        f(block, i, j, total);
    }
}

// Where the up to 16 JB rows of activations come from, 16 at a time.
template <class T, int JB> struct ThinFrom {
    typename ThinRows<T>::From of[JB];
    __device__ __forceinline__ ThinFrom(const T *first, int64_t stride, int64_t rows) : ThinFrom(first, stride, rows, std::make_integer_sequence<int, JB>{}) {}
private:
    template <int... B>
    __device__ __forceinline__ ThinFrom(const T *first, int64_t stride, int64_t rows, std::integer_sequence<int, B...>)
        : of{typename ThinRows<T>::From(first + (16 * B < rows ? 16 * B : rows - 1) * stride, stride, 16 * B < rows ? rows - 1 - 16 * B : 0)...}
    {
    }
};

// A staged operand, as parts.
template <class T, int P> __device__ __forceinline__ void thin_parts(const f32x4 *slot, const SplitConst &sc, bf16x8 (&out)[P])
{
    T v[8];
    ThinRows<T>::read(slot, v);
    to_parts<T, P>(v, sc, out);
}

// calls f(b, parts) for each of the JB operands of 16 rows, the first of which is staged in `slot`
template <class T, int JB, class F> __device__ __forceinline__ void each_thin_row(const ThinRows<T> (&r)[JB], f32x4 *slot, const SplitConst &sc, F f)
{
#pragma unroll
    for (int b = 0; b < JB; ++b) {
        if (b > 0) {
            wave_sync();
            r[b].stage(slot);
            wave_sync();
        }
        bf16x8 parts[kParts<T>];
        thin_parts<T, kParts<T>>(slot, sc, parts);
        f(b, parts);
    }
}

// Which 16 (32) values of which particle a workgroup computes.
struct ThinGrid {
    int per_particle, of;
    __host__ ThinGrid(int64_t size, int o) : per_particle((int)((size + o - 1) / o)), of(o) {}
    __device__ __forceinline__ int particle() const { return blockIdx.x / per_particle; }
    __device__ __forceinline__ int64_t first() const { return (int64_t)(blockIdx.x % per_particle) * of; }
};

// The wave's whole steps, U at a time through load(u, k) and then use(u), u = 0 .. U - 1, those that are left over one by one; then the last step, if it
// is this wave's and not whole, through load_last(k) and use(0).
template <int U, class Load, class Last, class Use> __device__ __forceinline__ void thin_steps(int64_t K, Load load, Last load_last, Use use)
{
    const int wave = wave_of_block();
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
SVGD_THIN_KERNEL void thin_gate_up_kernel(FfnShape s, ThinGrid grid, Rows<const T> x, Params gate, Params up, float *h,
                                                                  float *g_out, float *u_out)
{
    constexpr int P = kParts<T>, U = 1, kPart = kThinPart<2 * JB, 3>;
    __shared__ f32x4 parts[kThinWaves * kPart];
    f32x4 *const slots = parts + wave_of_block() * kPart;
    const int particle = grid.particle();
    const int64_t i0 = grid.first(), last = s.hidden - 1 - i0;
    const ThinRows<float>::From wg(gate.p + particle * gate.stride + i0 * s.width, s.width, last), wu(up.p + particle * up.stride + i0 * s.width, s.width, last);
    const ThinFrom<T, JB> xr(x.p + particle * x.particle, x.row, s.rows);
    const SplitConst sc = split_const();
    ThinRows<float> g[U], u[U];
    ThinRows<T> r[U][JB];
    f32x4 c[2 * JB];
#pragma unroll
    for (int b = 0; b < 2 * JB; ++b) c[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    thin_steps<U>(
        s.width,
        [&](int q, int64_t k) {
            g[q].load(wg, k);
            u[q].load(wu, k);
#pragma unroll
            for (int b = 0; b < JB; ++b) r[q][b].load(xr.of[b], k);
        },
        [&](int64_t k) {
            g[0].load_last(wg, k, s.width);
            u[0].load_last(wu, k, s.width);
#pragma unroll
            for (int b = 0; b < JB; ++b) r[0][b].load_last(xr.of[b], k, s.width);
        },
        [&](int q) {
            wave_sync(); // (the step before has been read)
            g[q].stage(slots);
            u[q].stage(slots + kSlot);
            r[q][0].stage(slots + 2 * kSlot);
            wave_sync();
            bf16x8 gp[3], up_[3];
            thin_parts<float, 3>(slots, sc, gp);
            thin_parts<float, 3>(slots + kSlot, sc, up_);
            each_thin_row<T, JB>(r[q], slots + 2 * kSlot, sc, [&](int b, const bf16x8(&xp)[P]) {
                thin_product<3, P>(gp, xp, c[2 * b]);
                thin_product<3, P>(up_, xp, c[2 * b + 1]);
            });
        });
    join_waves<2 * JB, 2>(c, parts, kPart, [&](int b, int ii, int jj, const float (&v)[2]) {
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

template <class T, int JB> SVGD_THIN_KERNEL void thin_down_kernel(FfnShape s, ThinGrid grid, const float *h, Params down, Rows<T> y)
{
    constexpr int U = JB == 1 ? 2 : 4 / JB, kPart = kThinPart<JB, 2>;
    __shared__ f32x4 parts[kThinWaves * kPart];
    f32x4 *const slots = parts + wave_of_block() * kPart;
    const int particle = grid.particle();
    const int64_t i0 = grid.first();
    const ThinRows<float>::From w(down.p + particle * down.stride + i0 * s.hidden, s.hidden, s.width - 1 - i0);
    const ThinFrom<float, JB> hr(h + particle * s.rows * s.hidden_ld, s.hidden_ld, s.rows);
    const SplitConst sc = split_const();
    ThinRows<float> a[U], r[U][JB];
    f32x4 c[JB];
#pragma unroll
    for (int b = 0; b < JB; ++b) c[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    thin_steps<U>(
        s.hidden,
        [&](int q, int64_t k) {
            a[q].load(w, k);
#pragma unroll
            for (int b = 0; b < JB; ++b) r[q][b].load(hr.of[b], k);
        },
        [&](int64_t k) {
            a[0].load_last(w, k, s.hidden);
#pragma unroll
            for (int b = 0; b < JB; ++b) r[0][b].load_last(hr.of[b], k, s.hidden);
        },
        [&](int q) {
            wave_sync();
            a[q].stage(slots);
            r[q][0].stage(slots + kSlot);
            wave_sync();
            bf16x8 ap[3];
            thin_parts<float, 3>(slots, sc, ap);
            each_thin_row<float, JB>(r[q], slots + kSlot, sc, [&](int b, const bf16x8(&hp)[3]) { thin_product<3, 3>(ap, hp, c[b]); });
        });
    join_waves<JB, 1>(c, parts, kPart, [&](int b, int ii, int jj, const float (&v)[1]) {
        const int64_t j = b * 16 + jj;
        if (j < s.rows && i0 + ii < s.width) y.p[particle * y.particle + j * y.row + i0 + ii] = (T)v[0];
    });
}

template <class T, int ACT, int JB>
__global__ __launch_bounds__(kThinBlock) void thin_hidden_grad_kernel(FfnShape s, ThinGrid grid, Rows<const T> dy, Params down, const float *g,
                                                                      const float *u, float *dg, float *du)
{
    constexpr int P = kParts<T>, U = 2, kPart = kThinPart<2 * JB, 0>;
    __shared__ f32x4 parts[kThinWaves * kPart];
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
    join_waves<2 * JB, 1>(c, parts, kPart, [&](int b, int ii, int jj, const float (&v)[1]) {
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
    constexpr int U = 2, kPart = kThinPart<2 * JB, 0>;
    __shared__ f32x4 parts[kThinWaves * kPart];
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
    join_waves<2 * JB, 1>(c, parts, kPart, [&](int b, int ii, int jj, const float (&v)[1]) {
        const int64_t j = (b >> 1) * 16 + jj, col = i0 + 2 * ii + (b & 1);
        if (j < s.rows && col < s.width) dx.p[particle * dx.particle + j * dx.row + col] = (T)v[0];
    });
}

} // namespace svgd
