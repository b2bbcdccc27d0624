// What the attention kernels share: arguments, tiles of keys or rows in LDS, operands of the matrix instructions, masks.
//
// Queries of the heads that share a key head are one list of rows: row r is query r / group of head r % group of those.  A wave holds rows (or keys) of its own as the
// B operand of the matrix instructions, 16 to a block, and streams the others past them as A: the results then have a row of the wave's own per lane (lane % 16), and of the streamed
// ones 4 (lane / 16) + 0 .. 3 of every 16.  Softmax statistics are one register per lane, and probabilities are, as they come, the B operand of the next product: two blocks of 16
// make a step of 32 whose k are ordered as k_of says, in A as in B.
#pragma once
#include "../../include/svgd_attention.h"
#include "layer_common.hpp"

namespace svgd {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
constexpr int kTileRows = 64; // streamed rows (or keys) in LDS at a time
constexpr int kAttnWaves = 4, kAttnBlock = 64 * kAttnWaves;
constexpr int kMaxStart = 1 << 28;

template <class T> struct Heads {
    T *p;
    int64_t particle, batch, token, head;
    __device__ __forceinline__ T *at(int i, int b, int h) const { return p + i * particle + b * batch + h * head; }
};

struct AttnArgs {
    int n, batch, heads, kv, group, dim;
    int t, s, rows; // rows = t group: of one key head
    uint32_t group_mul;
    int causal;
    float scale, cap;
    const float *slopes;
    int64_t slopes_stride;
    const int32_t *starts, *lengths, *documents, *prefix;
    int tiles, splits, per_split; // tiles of a workgroup's own rows; parts of the streamed ones, and tiles of 64 of each part
    int per_die, total;           // workgroups
    __device__ __forceinline__ int query(int r) const { return group == 1 ? r : (int)__umulhi((uint32_t)r, group_mul); } // exact: r group < 2^32
    __device__ __forceinline__ int64_t line(int i, int b, int h, int query) const { return ((int64_t)(i * batch + b) * heads + h) * t + query; }
};

// Which particle, sequence, key head, tile and part a workgroup has.  Workgroups go round the eight dies in turn; a die gets tiles that follow one another, which share keys in its L2.
struct AttnBlock {
    int particle, batch, head, tile, part;
    bool any;
    __device__ __forceinline__ AttnBlock(const AttnArgs &a)
    {
        int id = (int)(blockIdx.x & 7) * a.per_die + (int)(blockIdx.x >> 3);
        any = id < a.total;
        part = id % a.splits;
        id /= a.splits;
        tile = id % a.tiles;
        id /= a.tiles;
        head = id % a.kv;
        id /= a.kv;
        batch = id % a.batch;
        particle = id / a.batch;
    }
};

// ---------------------------------------------------------------------------------------------
// operands
// ---------------------------------------------------------------------------------------------
template <class T> struct FragOf {
    typedef T type __attribute__((ext_vector_type(8)));
};
template <class T> using Frag = typename FragOf<T>::type; // eight values of k of one row, lane l: row l % 16, group l / 16 of k

__device__ __forceinline__ f32x4 mma(Frag<bf16_t> a, Frag<bf16_t> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(Frag<f16_t> a, Frag<f16_t> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(Frag<float> a, Frag<float> b, f32x4 c)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// Eight values from memory, those from `left` on 0 and not read.
template <class T> __device__ __forceinline__ Frag<T> load_frag(const T *p, int left)
{
    Frag<T> f;
    constexpr int W = 16 / sizeof(T);
    if (left >= 8) {
#pragma unroll
        for (int q = 0; q < 8; q += W) {
            const typename Pack<T, W>::raw r = *reinterpret_cast<const typename Pack<T, W>::type *>(p + q);
#pragma unroll
            for (int e = 0; e < W; ++e) f[q + e] = r[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            f[e] = (T)0.f;
            if (e < left) f[e] = p[e];
        }
    }
    return f;
}

// 64 rows of up to 32 KD values in LDS, as they are in memory; 16 bytes between rows, so that 16 rows at the same place meet in no bank.
template <class T, int KD> struct Tile64 {
    static constexpr int VEC = 16 / sizeof(T), kLd = 32 * KD + VEC, kSize = kTileRows * kLd, kChunks = 32 * KD / VEC, N = kTileRows * kChunks / kAttnBlock;
    typedef typename Pack<T, VEC>::raw raw;
    raw v[N];
    // row(i): where row i of the tile starts; rows from `count` on are 0 and not read
    template <class F> __device__ __forceinline__ void load(int count, int dim, F row)
    {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int k = threadIdx.x + kAttnBlock * u, i = k / kChunks, c = (k - i * kChunks) * VEC;
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[u][e] = (T)0.f;
            if (i < count && c < dim) {
                const T *const p = row(i) + c;
                if (c + VEC <= dim) {
                    v[u] = *reinterpret_cast<const typename Pack<T, VEC>::type *>(p);
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (c + e < dim) v[u][e] = p[e];
                }
            }
        }
    }
    __device__ __forceinline__ void store(T *lds) const
    {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int k = threadIdx.x + kAttnBlock * u, i = k / kChunks, c = (k - i * kChunks) * VEC;
            *reinterpret_cast<raw *>(lds + i * kLd + c) = v[u];
        }
    }
    // operand of rows row .. row + 15, values col .. col + 31
    static __device__ __forceinline__ Frag<T> rows(const T *lds, int row, int col)
    {
        const int lane = threadIdx.x & 63;
        const T *const p = lds + (row + (lane & 15)) * kLd + col + 8 * (lane >> 4);
        Frag<T> f;
#pragma unroll
        for (int q = 0; q < 8; q += VEC) {
            const raw r = *reinterpret_cast<const raw *>(p + q);
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[q + e] = r[e];
        }
        return f;
    }
    // operand of values col .. col + 15 (its rows), rows row .. row + 31 (its k, ordered 4 g + 0 .. 3, 16 + 4 g + 0 .. 3)
    static __device__ __forceinline__ Frag<T> columns(const T *lds, int row, int col)
    {
        const int lane = threadIdx.x & 63, g = lane >> 4;
        Frag<T> f;
        if constexpr (sizeof(T) == 2) {
            // (16 lanes read 4 rows of 16 values, a lane the four values of the rows' column lane % 16)
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 lds16x4;
            typedef T t4 __attribute__((ext_vector_type(4)));
            const T *const p = lds + (row + 4 * g + ((lane & 15) >> 2)) * kLd + col + 4 * (lane & 3);
            const t4 lo = __builtin_bit_cast(t4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16x4 *)p));
            const t4 hi = __builtin_bit_cast(t4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16x4 *)(p + 16 * kLd)));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[e] = lo[e];
                f[4 + e] = hi[e];
            }
        } else {
            const T *const p = lds + (row + 4 * g) * kLd + col + (lane & 15);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = p[((e & 3) + 16 * (e >> 2)) * kLd];
        }
        return f;
    }
};

// Two results of 16 streamed rows each as a B operand.
template <class T> __device__ __forceinline__ Frag<T> as_operand(f32x4 a, f32x4 b)
{
    Frag<T> f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[e] = (T)a[e];
        f[4 + e] = (T)b[e];
    }
    return f;
}

// The largest of the four lanes l, l ^ 16, l ^ 32, l ^ 48, in all of them.
__device__ __forceinline__ float max_over_rows(float v)
{
    const unsigned u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const float s = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const unsigned w = __float_as_uint(s);
    const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// tanh: for 16-bit activations from one exponential, off by 2^-23 or so of 1; for fp32 the library's.
template <class T> __device__ __forceinline__ float tanh_of(float x)
{
    if constexpr (sizeof(T) == 4) return tanhf(x);
    else return 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * (2.f * kLog2e)));
}

// What a sequence's masks are.
struct Masks {
    int start, length, prefix;
    const int32_t *documents; // of the sequence
    __device__ __forceinline__ Masks(const AttnArgs &a, int b)
    {
        start = a.s - a.t;
        if (a.starts) start = min(max(a.starts[b], -kMaxStart), kMaxStart);
        length = a.lengths ? min(max(a.lengths[b], 0), a.s) : a.s;
        prefix = a.prefix ? min(a.prefix[b], a.s) : 0;
        documents = a.documents ? a.documents + (int64_t)b * a.s : nullptr;
    }
    // keys from here on are not seen from position p
    __device__ __forceinline__ int end(const AttnArgs &a, int p) const
    {
        if (documents && (p < 0 || p >= a.s)) return 0;
        return a.causal ? min(length, max(p + 1, prefix)) : length;
    }
    __device__ __forceinline__ int document(const AttnArgs &a, int p) const { return documents && p >= 0 && p < a.s ? documents[p] : 0; }
};

// Narrows the streamed places [lo, hi) to those from the first to the last that may share a document with one of the places [first, last]: all threads of the workgroup call it.
__device__ __forceinline__ void narrow(const int32_t *documents, int first, int last, int size, int *red, int &lo, int &hi)
{
    first = max(first, 0);
    last = min(last, size - 1);
    lo = max(lo, 0);
    hi = min(hi, size);
    if (threadIdx.x < 4) red[threadIdx.x] = threadIdx.x & 1 ? INT32_MIN : INT32_MAX;
    __syncthreads();
    for (int p = first + (int)threadIdx.x; p <= last; p += kAttnBlock) {
        atomicMin(&red[0], documents[p]);
        atomicMax(&red[1], documents[p]);
    }
    __syncthreads();
    const int least = red[0], most = red[1];
    int from = INT32_MAX, to = INT32_MIN;
    for (int j = lo + (int)threadIdx.x; j < hi; j += kAttnBlock) {
        const int d = documents[j];
        if (d >= least && d <= most) {
            from = min(from, j);
            to = max(to, j);
        }
    }
    if (to >= from) {
        atomicMin(&red[2], from);
        atomicMax(&red[3], to);
    }
    __syncthreads();
    lo = red[2];
    hi = red[3] == INT32_MIN ? lo : red[3] + 1;
    if (lo == INT32_MAX) lo = hi = 0;
}

// fp16 operands made of sums' terms (dz): scaled by a power of two that keeps the largest so far below 2^15, by wave.  Without it gradients below 6e-5 would lose their digits and those beyond 65,504 be infinite.
struct BlockScale {
    float scale = 0x1p100f;
    // the factor by which what was summed up so far has to be multiplied (mostly 1), given the lane's largest new magnitude
    __device__ __forceinline__ float take(float largest)
    {
#pragma unroll
        for (int m = 1; m < 16; m <<= 1) largest = fmaxf(largest, __shfl_xor(largest, m));
        largest = max_over_rows(largest);
        if (!(largest * scale > 32768.f)) return 1.f;
        const float next = ldexpf(1.f, min(max(14 - __builtin_amdgcn_frexp_expf(largest), -126), 100));
        const float factor = next / scale;
        scale = next;
        return factor;
    }
};

} // namespace svgd
