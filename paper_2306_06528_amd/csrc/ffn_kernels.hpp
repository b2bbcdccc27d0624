// The products of a gated feed-forward block and of its backward pass, for all particles in one launch each:
//     g = x Wg^T, u = x Wu^T, h = act(g) u                       gate_up_kernel   (the activation in its epilogue)
//     y = h Wd^T                                                 down_kernel
//     dh = dy Wd, dg = dh u act'(g), du = dh act(g)              hidden_grad_kernel (these in its epilogue)
//     dx = dg Wg + du Wu                                         gradients_kernel, input_grad_tile
//     dWg = dg^T x, dWu = du^T x, dWd = dy^T h                   gradients_kernel, weight_grad_tile
//
// All of them are one tile product, C[j][i] = sum_k A[i][k] B[j][k], 256 x 128 values of C (i x j) per workgroup of four waves of 64 x 128, or
// less where there are few tiles (ffn_launch.hpp).  Operands are fp32 or 16 bits wide in memory; on their way into LDS they become bf16 parts whose sum is the value
// EXACTLY (split3: three parts of an fp32 value, two of an fp16 one, one of a bf16 one), and the matrix cores
// add up the products of parts that are not below 2^-24 of the whole: six for two fp32 operands, five for fp32 and fp16, three for fp32 and bf16.  That is
// the accuracy of fp32 products at 2.5 PFLOP/s / 6 (5, 3), where the fp32 matrix instructions end at 157 TFLOP/s; and
// since each part is read from LDS once for several products, LDS keeps up with half the traffic a
// plain bf16 product needs.  The matrix cores bound the large products: 8 x 4,096 x 1,024 x 2,730 bf16, forward and backward, are 6.60 TFLOP
// of theirs and take 5.65 to 5.76 ms, 1,145 to 1,170 TFLOP/s (a library's 8,192^3 bf16 product reaches 1,120 to 1,155 on the same card).
#pragma once
#include "ffn_rules.hpp"
#include "layer_common.hpp"

namespace svgd {

// A workgroup of W waves computes 64 W values of i and 16 NJ of j, each wave 64 of i and all of j.
template <int W, int NJ> struct Tile {
    static constexpr int kWaves = W, kBlocksJ = NJ, kThreads = 64 * W, kI = 64 * W, kJ = 16 * NJ;
    static constexpr int kPlane = kJ * 4; // 16-byte units of one part of B's rows
};

template <class T> constexpr int kParts = 3;
template <> inline constexpr int kParts<f16_t> = 2;
template <> inline constexpr int kParts<bf16_t> = 1;

// B's rows in LDS, one plane per part, each row four 16-byte units (8 values of k).  Two rows share 128 bytes; which half a row takes
// and where its units lie in it is permuted so that neither 8 rows in succession nor 8 every-second rows (what eight
// lanes write at a time) meet in a bank.
__device__ __forceinline__ int unit_of(int row, int kg) { return (row >> 1) * 8 + (((row ^ (row >> 3)) & 1) << 2) + (kg ^ ((row >> 1) & 3)); }

// The order of k within a step: group g of 8 values that one lane hands to a matrix instruction has 4 g .. 4 g + 3 and 16 more than
// these, in A as in B.  Four lanes then read 64 bytes of an fp32 row side by side.
__device__ __forceinline__ constexpr int k_of(int g, int e) { return 4 * g + (e & 3) + 16 * (e >> 2); }

// The wave's number, known to be the same in all its lanes.
__device__ __forceinline__ int wave_of_block() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

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

// A, whose rows no other wave of the workgroup needs, goes from memory to the registers of the matrix instructions without LDS.
// Instruction block ib (of four) has rows 4 quad(m) + ib of the wave's 64, m = 0 .. 15; lane l holds m = l % 16, k of group l / 16.  Since a
// lane's results are those of m = 4 (l / 16) + r, r = 0 .. 3, their quads are l / 16 + 4 r: four lanes have 16 results side by side, 64 bytes.
// `fetch` brings a whole step and has no branch, so that it can lie among the matrix instructions; `fetch_any` brings
// any step, value by value, columns from K on as 0 and unread.

__device__ __forceinline__ int quad_of_lane() { return ((threadIdx.x & 15) >> 2) + 4 * (threadIdx.x & 3); }

// K contiguous in memory, fp32.  The vector memory unit joins what 16 lanes in a row read, and those of the matrix instructions'
// layout read 16 rows: 64 accesses for each load, which kept it busy 86 % of the time.  So eight lanes read 128 bytes of a row, and
// the values change lanes in the wave's own part of LDS, kScratch floats, as they are.
template <int P, int STEP> struct RowsOfA { // STEP: 2 where the groups of 8 rows are of gate and up by turns
    const float *from[2]; // of even and of odd groups of 8 rows: the wave's first row there
    int last;             // rows beyond this one: this one again
    uint32_t row_bytes;   // below 2^24
    f32x4 v[8];
    static constexpr bool narrow = false, kStaged = true;
    __device__ __forceinline__ RowsOfA(const float *even, const float *odd, int64_t rows_left, int64_t width)
        : last(rows_left < 64 ? (int)rows_left - 1 : 63), row_bytes((uint32_t)width * 4)
    {
        from[0] = even;
        from[1] = odd;
    }
    static __device__ __forceinline__ int row_of(int n) { return 8 * n + ((threadIdx.x & 63) >> 3); }
    static __device__ __forceinline__ int place(int row, int piece) { return row * 8 + (piece ^ (((row >> 4) & 3) | (row & 4))); } // in 16 bytes
    // Two instructions each time rather than eight registers: `row` is the lane's, hidden from the compiler.
    __device__ __forceinline__ uint32_t offset(int n, int row) const
    {
        const int r = 8 * (n / STEP) + row;
        return __umul24(r < last ? r : last, row_bytes) + 16 * (threadIdx.x & 7);
    }
    __device__ __forceinline__ void fetch(int64_t k0)
    {
        int row = (threadIdx.x & 63) >> 3;
        asm volatile("" : "+v"(row));
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const char *const p = reinterpret_cast<const char *>(from[n & (STEP - 1)] + k0);
            v[n] = *reinterpret_cast<const f32x4u *>(p + offset(n, row));
        }
    }
    __device__ __forceinline__ void fetch_any(int64_t k0, int64_t K)
    {
        const int64_t k = k0 + 4 * (threadIdx.x & 7);
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const float *const row = reinterpret_cast<const float *>(reinterpret_cast<const char *>(from[n & (STEP - 1)]) + offset(n, (threadIdx.x & 63) >> 3)) - 4 * (threadIdx.x & 7);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = row[k + e < K ? k + e : K - 1];
                v[n][e] = k + e < K ? x : 0.f;
            }
        }
    }
    __device__ __forceinline__ void leave_out(int count) // the step's first `count` columns count as 0
    {
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (4 * (int)(threadIdx.x & 7) + e < count) v[n][e] = 0.f;
    }
    __device__ __forceinline__ void stage(float *scratch) const
    {
        f32x4 *const s = reinterpret_cast<f32x4 *>(scratch);
        wave_sync(); // (the step before has been read)
#pragma unroll
        for (int n = 0; n < 8; ++n) s[place(row_of(n), threadIdx.x & 7)] = v[n];
        wave_sync();
    }
    __device__ __forceinline__ void parts(int ib, const SplitConst &sc, bf16x8 (&out)[P], const float *scratch) const
    {
        const f32x4 *const s = reinterpret_cast<const f32x4 *>(scratch);
        const int row = 4 * quad_of_lane() + ib, g = (threadIdx.x & 63) >> 4;
        split_parts<P>(s[place(row, g)], s[place(row, g + 4)], sc, out);
    }
};

// The rows contiguous in memory, `count` of them, k after k `stride` apart: a lane's four rows are one load.  Where
// these end beyond the last row they are the last four instead (quad_of says which).
constexpr int64_t kFarStride = (int64_t)1 << 22;
__device__ __forceinline__ int64_t quad_of(int64_t i, int64_t count) { return i + 4 <= count ? i : count - 4; }

template <class T, int P> struct ColumnsOfA {
    const T *base;   // row 0
    int64_t stride;  // beyond kFarStride every step goes the slow way: a lane's offset is to fit 32 bits
    uint32_t column; // the lane's first row (fewer than four rows: the first one)
    int rows;        // of them, if they are fewer than four; otherwise 4
    bool narrow;
    static constexpr bool kStaged = false;
    typename Pack<T, 4>::raw v[8];
    __device__ __forceinline__ ColumnsOfA(const T *b, int64_t s, int64_t first, int64_t count)
        : base(b), stride(s), column(count < 4 ? 0 : (uint32_t)quad_of(first + 4 * quad_of_lane(), count)), rows(count < 4 ? (int)count : 4),
          narrow(count < 4 || s > kFarStride)
    {
    }
    __device__ __forceinline__ void fetch(int64_t k0)
    {
        const int g = (threadIdx.x & 63) >> 4;
        const uint32_t offset = (column + 4 * g * (uint32_t)stride) * (uint32_t)sizeof(T);
        const char *const from = reinterpret_cast<const char *>(base + k0 * stride);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = *reinterpret_cast<const typename Pack<T, 4>::type *>(from + k_of(0, e) * stride * (int64_t)sizeof(T) + offset);
    }
    __device__ __forceinline__ void fetch_any(int64_t k0, int64_t K)
    {
        const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int64_t k = k0 + k_of(g, e);
            const T *const line = base + (k < K ? k : K - 1) * stride + column;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const T x = line[t < rows ? t : rows - 1];
                v[e][t] = k < K ? x : (T)0.f;
            }
        }
    }
    __device__ __forceinline__ void leave_out(int count)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (k_of((threadIdx.x & 63) >> 4, e) < count) v[e][t] = (T)0.f;
    }
    __device__ __forceinline__ void stage(float *) const {}
    __device__ __forceinline__ void parts(int ib, const SplitConst &sc, bf16x8 (&out)[P], const float *) const
    {
        T x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = v[e][ib];
        to_parts<T, P>(x, sc, out);
    }
};

// B goes through LDS, each thread bringing 8 values of k of some rows.  K contiguous in memory: rows tid / 4 + 16 W t, again from the
// first one on where there are not so many (twice the same values to the same place, but no branch).
template <class TL, class T, int P> struct RowsOfB {
    static constexpr int N = (TL::kBlocksJ + TL::kWaves - 1) / TL::kWaves;
    static __device__ __forceinline__ int row_of(int t)
    {
        const int r = (threadIdx.x >> 2) + 16 * TL::kWaves * t;
        return N * TL::kWaves == TL::kBlocksJ || r < TL::kJ ? r : r - TL::kJ;
    }
    const T *base;  // the tile's first row
    int64_t stride; // beyond kFarStride the slow way, as above
    int last;       // rows beyond this one: this one again
    bool narrow;
    T v[N][8];
    __device__ __forceinline__ RowsOfB(const T *b, int64_t s, int64_t rows_left)
        : base(b), stride(s), last(rows_left < TL::kJ ? (int)rows_left - 1 : TL::kJ - 1), narrow(s > kFarStride)
    {
    }
    __device__ __forceinline__ int source(int t) const { return row_of(t) < last ? row_of(t) : last; }
    __device__ __forceinline__ void fetch(int64_t k0)
    {
        const int g = threadIdx.x & 3;
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const uint32_t offset = ((uint32_t)source(t) * (uint32_t)stride + k_of(g, 0)) * (uint32_t)sizeof(T);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const char *const from = reinterpret_cast<const char *>(base + k0 + k_of(0, 4 * q));
                const typename Pack<T, 4>::raw r = *reinterpret_cast<const typename Pack<T, 4>::type *>(from + offset);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[t][4 * q + e] = r[e];
            }
        }
    }
    __device__ __forceinline__ void fetch_any(int64_t k0, int64_t K)
    {
        const int g = threadIdx.x & 3;
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t k = k0 + k_of(g, e);
                const T x = base[source(t) * stride + (k < K ? k : K - 1)];
                v[t][e] = k < K ? x : (T)0.f;
            }
    }
    __device__ __forceinline__ void store(bf16x8 *lds, const SplitConst &sc) const
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            bf16x8 parts[P];
            to_parts<T, P>(v[t], sc, parts);
            const int u = unit_of(row_of(t), threadIdx.x & 3);
#pragma unroll
            for (int p = 0; p < P; ++p) lds[p * TL::kPlane + u] = parts[p];
        }
    }
};

// Rows contiguous, `count` of them, k after k `stride` apart: two rows, the tile's 2 l and 2 l + 1, and one group of 8 values of k at a
// time.  A pair that ends beyond the last row is loaded one row earlier; its first row is then the second one loaded.
template <class TL, class T, int P> struct ColumnsOfB {
    static constexpr int kPairs = TL::kJ / 2, kAtATime = TL::kThreads / kPairs, N = (4 + kAtATime - 1) / kAtATime;
    static_assert(kAtATime >= 1, "a thread for every pair");
    const T *base;   // row 0
    int64_t stride;  // beyond kFarStride the slow way: a thread's offset is to fit 32 bits
    uint32_t column; // the first row of the thread's pair
    bool late, single, narrow;
    T v[N][2][8];
    __device__ __forceinline__ ColumnsOfB(const T *b, int64_t s, int64_t first, int64_t count)
        : base(b), stride(s), single(count < 2), narrow(count < 2 || s > kFarStride)
    {
        const int64_t j = first + row();
        late = j + 2 > count && !single;
        column = single ? 0 : (uint32_t)(late ? count - 2 : j);
    }
    static __device__ __forceinline__ int row() { return 2 * (threadIdx.x % kPairs); }
    static __device__ __forceinline__ int group(int t) { return (threadIdx.x / kPairs + t * kAtATime) & 3; } // (beyond the fourth: again)
    __device__ __forceinline__ void fetch(int64_t k0)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const uint32_t offset = (column + 4 * group(t) * (uint32_t)stride) * (uint32_t)sizeof(T);
            const char *const from = reinterpret_cast<const char *>(base + k0 * stride);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const typename Pack<T, 2>::raw x =
                    *reinterpret_cast<const typename Pack<T, 2>::type *>(from + k_of(0, e) * stride * (int64_t)sizeof(T) + offset);
                v[t][0][e] = x[0];
                v[t][1][e] = x[1];
            }
        }
    }
    __device__ __forceinline__ void fetch_any(int64_t k0, int64_t K)
    {
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t k = k0 + k_of(group(t), e);
                const T *const line = base + (k < K ? k : K - 1) * stride + column;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const T x = line[single ? 0 : q];
                    v[t][q][e] = k < K ? x : (T)0.f;
                }
            }
    }
    __device__ __forceinline__ void store(bf16x8 *lds, const SplitConst &sc) const
    {
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                T x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = q == 0 && late ? v[t][1][e] : v[t][q][e];
                bf16x8 parts[P];
                to_parts<T, P>(x, sc, parts);
                const int u = unit_of(row() + q, group(t));
#pragma unroll
                for (int p = 0; p < P; ++p) lds[p * TL::kPlane + u] = parts[p];
            }
    }
};

// The wave's 64 x 16 NJ values of C: in block (ib, jb) value r of lane l is i = 4 (l / 16) + 16 r + ib, j = 16 jb + l % 16.
template <int NJ> struct Acc {
    f32x4 c[4][NJ];
    __device__ __forceinline__ Acc()
    {
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int b = 0; b < NJ; ++b) c[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
};

// Adds the product over the columns from begin (a multiple of kTileK) to end to acc.  Products of parts pa, pb with pa + pb beyond the last of three are below 2^-24
// of the whole and left out; of two fp16 operands all four are there.  While the matrix cores work on a step, the next one's rows of B go to the
// other half of LDS and those of A are split into the registers of the last columns' blocks as these get free, and the rows of the
// step after it are on their way: one barrier per step.
// lds: 2 * PB * kPlane units; scratch: the wave's own kScratch floats.
// BACK: the last step, if it is not whole, begins further back, where it is, and what it has in common with the step before counts as 0: loaded like any other (otherwise value by value, behind
// the others).
constexpr int kScratch = 64 * kTileK; // 64 rows of a step of A; 16 rows of 68 values of C
template <class TL, int PA, int PB, bool BACK = false, class LA, class LB>
__device__ __forceinline__ void tile_product(LA &a, LB &b, int64_t begin, int64_t K, Acc<TL::kBlocksJ> &acc, bf16x8 *lds, float *scratch)
{
    if (begin >= K) return;
    constexpr int kOrder = PA == 3 || PB == 3 ? 2 : PA + PB - 2, NJ = TL::kBlocksJ, kStage = PB * TL::kPlane;
    constexpr int kLast = NJ <= 2 ? 1 : NJ <= 4 ? 2 : PB == 3 ? 1 : 2; // columns that go block of A by block of A: as many as there are registers for
    // Whether a step's rows are fetched during the whole step before it, or while it goes on: the former where there are registers for it;
    // in large tiles not if A takes the detour through LDS (large bf16 block: hidden_grad_kernel 705 us, otherwise 727, but
    // gate_up_kernel 1179 and 1096; tiles of 64 x 32: 1 x 500 x 256 x 700 fp32 forward 25.0 and 27.0).
    constexpr bool kAhead = NJ <= 4 || (!LA::kStaged && !(PA == 3 && PB == 3));
    static_assert(kLast < NJ, "columns to begin with");
    const SplitConst sc = split_const();
    const int lane = threadIdx.x & 63;
    const int frag = unit_of(lane & 15, lane >> 4);
    bf16x8 fa[4][PA];
    int stage = 0;
    const auto columns = [&](int first, int last) {
#pragma unroll
        for (int jb = first; jb < last; ++jb) {
            bf16x8 fb[PB];
#pragma unroll
            for (int p = 0; p < PB; ++p) fb[p] = lds[stage + p * TL::kPlane + jb * 64 + frag];
#pragma unroll
            for (int pa = 0; pa < PA; ++pa)
#pragma unroll
                for (int pb = 0; pb < PB; ++pb)
                    if (pa + pb <= kOrder) {
#pragma unroll
                        for (int ib = 0; ib < 4; ++ib)
                            acc.c[ib][jb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[ib][pa], fb[pb], acc.c[ib][jb], 0, 0, 0);
                    }
        }
    };
    const bool back = BACK && K >= kTileK;
    const int64_t whole = a.narrow || b.narrow ? begin : (back ? K + kTileK - 1 : K) / kTileK * kTileK;
    if (whole > begin) {
        const int64_t last = back ? K - kTileK : whole - kTileK; // (what is fetched ahead of the end is the last step again)
        b.fetch(BACK && last < begin ? last : begin);
        a.fetch(BACK && last < begin ? last : begin);
        __syncthreads(); // (an earlier product's last step has been read)
        b.store(lds, sc);
        if (BACK && begin + kTileK > K) a.leave_out((int)(begin + kTileK - K));
        a.stage(scratch);
#pragma unroll
        for (int ib = 0; ib < 4; ++ib) a.parts(ib, sc, fa[ib], scratch);
        if constexpr (kAhead) {
            b.fetch(begin + kTileK < last ? begin + kTileK : last);
            a.fetch(begin + kTileK < last ? begin + kTileK : last);
        }
        __syncthreads();
        // (the scheduling barriers: the compiler would move the loads down to where their values are needed)
        for (int64_t k0 = begin + kTileK; k0 < whole; k0 += kTileK) {
            const int64_t next = k0 + kTileK < last ? k0 + kTileK : last;
            if constexpr (kAhead) {
                b.store(lds + (kStage - stage), sc);
                b.fetch(next);
                __builtin_amdgcn_sched_barrier(0);
                columns(0, NJ - kLast);
                if (BACK && k0 + kTileK > K) a.leave_out((int)(k0 + kTileK - K));
                if constexpr (LA::kStaged) {
                    a.stage(scratch);
                    a.fetch(next);
                }
            } else {
                b.fetch(BACK && last < k0 ? last : k0);
                __builtin_amdgcn_sched_barrier(0);
                columns(0, NJ / 2 - 1);
                b.store(lds + (kStage - stage), sc);
                __builtin_amdgcn_sched_barrier(0);
                a.fetch(BACK && last < k0 ? last : k0);
                __builtin_amdgcn_sched_barrier(0);
                columns(NJ / 2 - 1, NJ - kLast);
                __builtin_amdgcn_sched_barrier(0);
                if (BACK && k0 + kTileK > K) a.leave_out((int)(k0 + kTileK - K));
                a.stage(scratch);
            }
            bf16x8 fb[kLast][PB];
#pragma unroll
            for (int q = 0; q < kLast; ++q)
#pragma unroll
                for (int p = 0; p < PB; ++p) fb[q][p] = lds[stage + p * TL::kPlane + (NJ - kLast + q) * 64 + frag];
#pragma unroll
            for (int ib = 0; ib < 4; ++ib) {
#pragma unroll
                for (int pa = 0; pa < PA; ++pa)
#pragma unroll
                    for (int pb = 0; pb < PB; ++pb)
                        if (pa + pb <= kOrder) {
#pragma unroll
                            for (int q = 0; q < kLast; ++q)
                                acc.c[ib][NJ - kLast + q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[ib][pa], fb[q][pb], acc.c[ib][NJ - kLast + q], 0, 0, 0);
                        }
                a.parts(ib, sc, fa[ib], scratch);
            }
            if constexpr (kAhead && !LA::kStaged) a.fetch(next);
            stage = kStage - stage;
            __syncthreads();
        }
        columns(0, NJ);
    }
#pragma unroll 1
    for (int64_t k0 = whole; k0 < K; k0 += kTileK) {
        b.fetch_any(k0, K);
        a.fetch_any(k0, K);
        __syncthreads();
        stage = 0;
        b.store(lds, sc);
        a.stage(scratch);
#pragma unroll
        for (int ib = 0; ib < 4; ++ib) a.parts(ib, sc, fa[ib], scratch);
        __syncthreads();
        columns(0, NJ);
    }
}

// Which tile a workgroup computes, over which part of the columns.  Workgroups go round the eight dies in turn: every die gets
// tiles that follow one another, so that the operands they share meet in its L2; and they follow one another in blocks of kBand tiles of j.
// Where there are few tiles the columns are split into `splits` parts of `per` columns: the parts' sums are added up afterwards,
// in order (reduce_rows_kernel, reduce_params_kernel).
constexpr int kBand = 8;
struct TileGrid {
    int ti, tj, splits, per_die, total;
    int64_t per, columns;
    __host__ TileGrid() : ti(0), tj(0), splits(1), per_die(0), total(0), per(0), columns(0) {}
    __host__ TileGrid(int n, int64_t i, int64_t j, int64_t cols, int parts) : ti((int)i), tj((int)j), splits(parts), columns(cols)
    {
        per = ((cols + parts - 1) / parts + kTileK - 1) / kTileK * kTileK;
        total = (int)(n * i * j * parts); // (the plan has seen to it that a launch takes them)
        per_die = (total + kDies - 1) / kDies;
    }
    __host__ int blocks() const { return per_die * kDies; }
    // false: nothing to do
    __device__ __forceinline__ bool at(int block, int &particle, int &part, int &i, int &j) const
    {
        const int id = (block % kDies) * per_die + block / kDies;
        if (id >= total) return false;
        const int each = ti * tj, p = id / each, r = id - p * each;
        particle = p / splits;
        part = p - particle * splits;
        const int band = r / (ti * kBand), left = r - band * ti * kBand;
        const int high = tj - band * kBand < kBand ? tj - band * kBand : kBand;
        i = left / high;
        j = band * kBand + left - i * high;
        return true;
    }
    __device__ __forceinline__ int64_t begin(int part) const { return part * per; }
    __device__ __forceinline__ int64_t end(int part) const { return (part + 1) * per < columns ? (part + 1) * per : columns; } // (may lie before begin)
};

template <int ACT> __device__ __forceinline__ void activate(float g, float &a, float &slope)
{
    if constexpr (ACT == SVGD_SILU) {
        const float s = 1.f / (1.f + expf(-g));
        a = g * s;
        slope = s * (1.f + g * (1.f - s));
    } else {
        const float cdf = 0.5f * erfcf(g * -0.70710678118654752f); // (1 + erf has no digits left below -5)
        a = g * cdf;
        slope = cdf + g * 0.39894228040143268f * expf(-0.5f * g * g);
    }
}

struct FfnShape {
    int n;
    int64_t rows, width, hidden, hidden_ld, width_ld; // *_ld: row stride of g, u, h, dg, du in the buffers; of partial sums of y and dx
};
template <class T> struct Rows {
    T *p;
    int64_t particle, row; // strides
};

// 16 columns j of the wave's C at a time go through its part of LDS, so that 16 lanes have 64 values of i of one j side by side.
constexpr int kScratchRow = 68; // floats from one j to the next: eight of them meet in no bank
template <int NJ> __device__ __forceinline__ void spread(const Acc<NJ> &acc, int jb, float *scratch)
{
    const int lane = threadIdx.x & 63;
    wave_sync();
#pragma unroll
    for (int r = 0; r < 4; ++r)
        *reinterpret_cast<f32x4 *>(scratch + (lane & 15) * kScratchRow + 4 * (lane >> 4) + 16 * r) =
            f32x4{acc.c[0][jb][r], acc.c[1][jb][r], acc.c[2][jb][r], acc.c[3][jb][r]};
    wave_sync();
}

// calls f(i, j, quad, first) for every four values of C that lie side by side: C[j][i .. i + 3], of which those before `first`
// are another lane's (COLUMNS, A's columns were loaded: at the end of the `count` values of i, see quad_of) and those from count on are not there.
template <class TL, bool COLUMNS, class F>
__device__ __forceinline__ void each_quad(const Acc<TL::kBlocksJ> &acc, int64_t i0, int64_t count, int64_t j0, float *scratch, F f)
{
    const int lane = threadIdx.x & 63;
    const int64_t i = i0 + 4 * (lane & 15);
#pragma unroll
    for (int jb = 0; jb < TL::kBlocksJ; ++jb) {
        spread(acc, jb, scratch);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int j = 4 * q + (lane >> 4);
            const f32x4 c = *reinterpret_cast<const f32x4 *>(scratch + j * kScratchRow + 4 * (lane & 15));
            if (i < count) f(COLUMNS && count >= 4 ? quad_of(i, count) : i, j0 + 16 * jb + j, c, i);
        }
    }
}

// Values c[0 .. 3] to p[0 .. 3], those before `skip` and from `left` on left out.
template <class T> __device__ __forceinline__ void store_quad(T *p, f32x4 c, int skip, int64_t left)
{
    if (skip == 0 && left >= 4) {
        const float v[4] = {c[0], c[1], c[2], c[3]};
        store_pack<T, 4>(p, 4, v);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e >= skip && e < left) p[e] = (T)c[e];
    }
}

#define SVGD_TILE_KERNEL __global__ __launch_bounds__(TL::kThreads) __attribute__((amdgpu_waves_per_eu(2)))

// Of a wave's 64 rows of A every other 8 are of gate and the next 8 of up, the same 32 of both, so that the wave has g and u of the same
// values.
template <class TL, class T, int ACT, bool SAVE>
SVGD_TILE_KERNEL void gate_up_kernel(FfnShape s, TileGrid grid, Rows<const T> x, Params gate, Params up, float *h, float *g_out, float *u_out)
{
    __shared__ bf16x8 lds[2 * kParts<T> * TL::kPlane];
    __shared__ float scratches[TL::kWaves][kScratch];
    float *const scratch = scratches[wave_of_block()];
    int particle, part, ti, tj;
    if (!grid.at(blockIdx.x, particle, part, ti, tj)) return;
    const T *const xs = x.p + particle * x.particle;
    const int lane = threadIdx.x & 63;
    const int64_t i0 = (int64_t)ti * (TL::kI / 2) + wave_of_block() * 32, j0 = (int64_t)tj * TL::kJ;
    const int64_t first = i0 < s.hidden ? i0 : s.hidden - 1;
    RowsOfA<3, 2> a(gate.p + particle * gate.stride + first * s.width, up.p + particle * up.stride + first * s.width, s.hidden - first, s.width);
    RowsOfB<TL, T, kParts<T>> b(xs + j0 * x.row, x.row, s.rows - j0);
    Acc<TL::kBlocksJ> acc;
    tile_product<TL, 3, kParts<T>>(a, b, 0, s.width, acc, lds, scratch);
    const int piece = lane & 7; // four values: in the wave's rows of C those of gate are 16 (piece / 2) + 4 (piece % 2) on, those of up 8 behind
    const int64_t i = i0 + 4 * piece;
#pragma unroll
    for (int jb = 0; jb < TL::kBlocksJ; ++jb) {
        spread(acc, jb, scratch);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int64_t j = j0 + 16 * jb + 8 * q + (lane >> 3);
            const float *const c = scratch + (8 * q + (lane >> 3)) * kScratchRow + 16 * (piece >> 1) + 4 * (piece & 1);
            const f32x4 g = *reinterpret_cast<const f32x4 *>(c), u = *reinterpret_cast<const f32x4 *>(c + 8);
            if (j >= s.rows || i >= s.hidden_ld) continue; // (the columns from hidden to hidden_ld are never used)
            const int64_t at = (particle * s.rows + j) * s.hidden_ld + i;
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float act, slope;
                activate<ACT>(g[e], act, slope);
                v[e] = act * u[e];
            }
            *reinterpret_cast<f32x4 *>(h + at) = v;
            if constexpr (SAVE) {
                *reinterpret_cast<f32x4 *>(g_out + at) = g;
                *reinterpret_cast<f32x4 *>(u_out + at) = u;
            }
        }
    }
}

// h, dg and du and the parameters that they meet are fp32 whatever the activations' type, and so are these products: two parts of each, which leave out
// 2^-16 of a product, would show in 16-bit results of sums that cancel, and the same row would come out differently beside 32 and beside 65 others.
constexpr int kHiddenParts = 3;

// partial: with more than one part, their sums [part][particle][row][width_ld]
template <class TL, class T> SVGD_TILE_KERNEL void down_kernel(FfnShape s, TileGrid grid, const float *h, Params down, Rows<T> y, float *partial)
{
    constexpr int P = kHiddenParts;
    __shared__ bf16x8 lds[2 * P * TL::kPlane];
    __shared__ float scratches[TL::kWaves][kScratch];
    float *const scratch = scratches[wave_of_block()];
    int particle, part, ti, tj;
    if (!grid.at(blockIdx.x, particle, part, ti, tj)) return;
    const float *const w = down.p + particle * down.stride, *const hs = h + particle * s.rows * s.hidden_ld;
    const int64_t i0 = (int64_t)ti * TL::kI, j0 = (int64_t)tj * TL::kJ, iw = i0 + wave_of_block() * 64;
    const int64_t first = iw < s.width ? iw : s.width - 1;
    RowsOfA<P, 1> a(w + first * s.hidden, w, s.width - first, s.hidden);
    RowsOfB<TL, float, P> b(hs + j0 * s.hidden_ld, s.hidden_ld, s.rows - j0);
    Acc<TL::kBlocksJ> acc;
    tile_product<TL, P, P>(a, b, grid.begin(part), grid.end(part), acc, lds, scratch);
    float *const sums = partial + ((int64_t)part * s.n + particle) * s.rows * s.width_ld;
    each_quad<TL, false>(acc, iw, s.width, j0, scratch, [&](int64_t i, int64_t j, f32x4 c, int64_t) {
        if (j >= s.rows) return;
        if (grid.splits > 1) *reinterpret_cast<f32x4 *>(sums + j * s.width_ld + i) = c; // (what is beyond the width is not used)
        else store_quad(y.p + particle * y.particle + j * y.row + i, c, 0, s.width - i);
    });
}

template <class TL, class T, int ACT>
SVGD_TILE_KERNEL void hidden_grad_kernel(FfnShape s, TileGrid grid, Rows<const T> dy, Params down, const float *g, const float *u, float *dg, float *du)
{
    __shared__ bf16x8 lds[2 * kParts<T> * TL::kPlane];
    __shared__ float scratches[TL::kWaves][kScratch];
    float *const scratch = scratches[wave_of_block()];
    int particle, part, ti, tj;
    if (!grid.at(blockIdx.x, particle, part, ti, tj)) return;
    const int64_t i0 = (int64_t)ti * TL::kI, j0 = (int64_t)tj * TL::kJ, iw = i0 + wave_of_block() * 64;
    const T *const dys = dy.p + particle * dy.particle;
    ColumnsOfA<float, 3> a(down.p + particle * down.stride, s.hidden, iw, s.hidden);
    RowsOfB<TL, T, kParts<T>> b(dys + j0 * dy.row, dy.row, s.rows - j0);
    Acc<TL::kBlocksJ> acc;
    tile_product<TL, 3, kParts<T>>(a, b, 0, s.width, acc, lds, scratch);
    each_quad<TL, true>(acc, iw, s.hidden, j0, scratch, [&](int64_t i, int64_t j, f32x4 c, int64_t) {
        if (j >= s.rows) return;
        // (two lanes may have values of the same places here, and then the same values)
        const int64_t at = (particle * s.rows + j) * s.hidden_ld + i;
        const f32x4 gv = *reinterpret_cast<const f32x4u *>(g + at), uv = *reinterpret_cast<const f32x4u *>(u + at);
        f32x4 dgv, duv;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float act, slope;
            activate<ACT>(gv[e], act, slope);
            dgv[e] = c[e] * uv[e] * slope;
            duv[e] = c[e] * act;
        }
        *reinterpret_cast<f32x4u *>(dg + at) = dgv;
        *reinterpret_cast<f32x4u *>(du + at) = duv;
    });
}

// A tile of dx.  The columns are those of gate and then those of up: with more than one part the first half of the parts is gate's.
template <class TL, class T>
__device__ __forceinline__ void input_grad_tile(const FfnShape &s, const TileGrid &grid, int block, const float *dg, const float *du, const Params &gate,
                                                const Params &up, const Rows<T> &dx, float *partial, bf16x8 *lds, float *scratch)
{
    constexpr int P = kHiddenParts;
    int particle, part, ti, tj;
    if (!grid.at(block, particle, part, ti, tj)) return;
    const int64_t i0 = (int64_t)ti * TL::kI, j0 = (int64_t)tj * TL::kJ, iw = i0 + wave_of_block() * 64;
    const int halves = grid.splits / 2, first_half = grid.splits > 1 ? part / halves : 0, last_half = grid.splits > 1 ? first_half : 1;
    const int sub = grid.splits > 1 ? part - first_half * halves : 0;
    Acc<TL::kBlocksJ> acc;
#pragma unroll 1
    for (int half = first_half; half <= last_half; ++half) {
        const float *const w = half ? up.p + particle * up.stride : gate.p + particle * gate.stride;
        const float *const d = (half ? du : dg) + particle * s.rows * s.hidden_ld;
        ColumnsOfA<float, P> a(w, s.width, iw, s.width);
        RowsOfB<TL, float, P> b(d + j0 * s.hidden_ld, s.hidden_ld, s.rows - j0);
        tile_product<TL, P, P>(a, b, grid.begin(sub), grid.end(sub), acc, lds, scratch);
    }
    float *const sums = partial + ((int64_t)part * s.n + particle) * s.rows * s.width_ld;
    each_quad<TL, true>(acc, iw, s.width, j0, scratch, [&](int64_t i, int64_t j, f32x4 c, int64_t first) {
        if (j >= s.rows) return;
        if (grid.splits > 1) store_quad(sums + j * s.width_ld + i, c, (int)(first - i), s.width - i);
        else store_quad(dx.p + particle * dx.particle + j * dx.row + i, c, (int)(first - i), s.width - i);
    });
}

// out[j][i] (+)= sum over the rows t of b[t][j] a[t][i], `wide` values of i and `high` of j, for one or two pairs (b, out).  The activations
// of the network, of which 16-bit ones have fewer parts, are a: SWAPPED stores out[i][j], so that this holds for all three gradients.
// partial: with more than one part, their sums [part][particle][which of the two][wide * high].
template <class TA, class TB> struct WeightGrad {
    TileGrid grid;
    int64_t wide, high;
    int tiles_high, outs; // tiles of j, of one pair; pairs
    Rows<const TA> a;
    Rows<const TB> b[2];
    Params out[2];
    float *partial;
};

template <class TL, bool SWAPPED, bool BACK = false, class TA, class TB>
__device__ __forceinline__ void weight_grad_tile(const WeightGrad<TA, TB> &w, int block, bool accumulate, bf16x8 *lds, float *scratch)
{
    constexpr int PA = kParts<TA>, PB = kParts<TB>;
    int particle, part, ti, tj;
    if (!w.grid.at(block, particle, part, ti, tj)) return;
    const int which = tj >= w.tiles_high;
    if (which) tj -= w.tiles_high;
    const Rows<const TB> b_rows = which ? w.b[1] : w.b[0];
    const bool split = w.grid.splits > 1;
    const int n = w.grid.total / (w.grid.ti * w.grid.tj * w.grid.splits);
    float *const out = split ? w.partial + (((int64_t)part * n + particle) * w.outs + which) * w.wide * w.high
                             : const_cast<float *>(which ? w.out[1].p + particle * w.out[1].stride : w.out[0].p + particle * w.out[0].stride);
    const bool add = accumulate && !split;
    const int64_t i0 = (int64_t)ti * TL::kI, j0 = (int64_t)tj * TL::kJ, iw = i0 + wave_of_block() * 64;
    ColumnsOfA<TA, PA> a(w.a.p + particle * w.a.particle, w.a.row, iw, w.wide);
    ColumnsOfB<TL, TB, PB> b(b_rows.p + particle * b_rows.particle, b_rows.row, j0, w.high);
    Acc<TL::kBlocksJ> acc;
    tile_product<TL, PA, PB, BACK>(a, b, w.grid.begin(part), w.grid.end(part), acc, lds, scratch);
    each_quad<TL, true>(acc, iw, w.wide, j0, scratch, [&](int64_t i, int64_t j, f32x4 c, int64_t first) {
        if (j >= w.high) return;
        const int skip = (int)(first - i);
        const int64_t left = w.wide - i;
        if (add || SWAPPED) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (e < skip || e >= left) continue;
                float *const p = out + (SWAPPED ? (i + e) * w.high + j : j * w.wide + i + e);
                *p = add ? c[e] + *p : c[e];
            }
        } else {
            store_quad(out + j * w.wide + i, c, skip, left);
        }
    });
}

// What a backward pass has to do once dg and du are there, none of which waits for another, in one launch: the tiles of dx, then those of
// dgate and dup, then those of ddown.
template <class TL, class T>
SVGD_TILE_KERNEL void gradients_kernel(FfnShape s, TileGrid input, const float *dg, const float *du, Params gate, Params up, Rows<T> dx, float *dx_partial,
                                       WeightGrad<T, float> gates, WeightGrad<T, float> down, bool accumulate)
{
    constexpr int P = kHiddenParts;
    __shared__ bf16x8 lds[2 * P * TL::kPlane];
    __shared__ float scratches[TL::kWaves][kScratch];
    float *const scratch = scratches[wave_of_block()];
    int block = blockIdx.x;
    if (block < input.per_die * kDies) {
        input_grad_tile<TL, T>(s, input, block, dg, du, gate, up, dx, dx_partial, lds, scratch);
        return;
    }
    block -= input.per_die * kDies;
    if (block < gates.grid.per_die * kDies) {
        weight_grad_tile<TL, false>(gates, block, accumulate, lds, scratch);
        return;
    }
    weight_grad_tile<TL, true>(down, block - gates.grid.per_die * kDies, accumulate, lds, scratch);
}

// y = the sum of the parts' sums, in order.
template <class T> __global__ __launch_bounds__(256) void reduce_rows_kernel(FfnShape s, const float *partial, int parts, Rows<T> y)
{
    const int64_t quads = s.width_ld / 4, k = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (k >= s.n * s.rows * quads) return;
    const int64_t line = k / quads, i = (k - line * quads) * 4, particle = line / s.rows, j = line - particle * s.rows;
    const int64_t each = s.n * s.rows * s.width_ld;
    const float *p = partial + line * s.width_ld + i;
    f32x4 total = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int part = 0; part < parts; ++part) total += *reinterpret_cast<const f32x4 *>(p + part * each);
    store_quad(y.p + particle * y.particle + j * y.row + i, total, 0, s.width - i);
}

// The same for gradients of parameters: `size` values of each of `outs` per particle.
static __global__ __launch_bounds__(256) void reduce_params_kernel(int n, int64_t size, int outs, const float *partial, int parts, Params out0, Params out1,
                                                            bool accumulate)
{
    const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x, each = n * outs * size;
    if (k >= each) return;
    float total = 0.f;
#pragma unroll 8
    for (int part = 0; part < parts; ++part) total += partial[part * each + k];
    const int64_t line = k / size, at = k - line * size, particle = line / outs;
    const Params &out = line - particle * outs ? out1 : out0;
    float *const p = const_cast<float *>(out.p) + particle * out.stride + at;
    *p = accumulate ? total + *p : total;
}

} // namespace svgd
