// What the attention kernels share: arguments, tiles of keys or rows in LDS, operands of the matrix instructions, masks.
//
// Queries of the heads that share a key head are one list of rows: row r is query r / group of head r % group of those.  A wave holds rows
// (or keys) of its own as the B operand of the matrix instructions, 16 to a block, and streams the others past them as A: the results then
// have a row of the wave's own per lane (lane % 16), and of the streamed ones 4 (lane / 16) + 0 .. 3 of every 16.  Softmax statistics are
// one register per lane, and probabilities are, as they come, the B operand of the next product: two blocks of 16 make a step of 32 whose k
// are ordered as k_of says, in A as in B.
#pragma once
#include "../../include/svgd_attention.h"
#include "attention_rules.hpp"
#include "layer_common.hpp"

namespace svgd {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
constexpr int kMaxStart = 1 << 28;
constexpr int64_t kMaxTokenStride = SVGD_ATTENTION_MAX_STRIDE; // (offsets within a tile fit 32 bits)

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
    int tiles, splits; // tiles of a workgroup's own rows; parts of the streamed ones
    int per_die, total;           // workgroups
    __device__ __forceinline__ int query(int r) const { return group == 1 ? r : (int)__umulhi((uint32_t)r, group_mul); } // exact: r group < 2^32
    __device__ __forceinline__ bool blind() const { return starts || lengths || t > s; } // there may be queries that see nothing
    __device__ __forceinline__ int64_t line(int i, int b, int h, int query) const { return ((int64_t)(i * batch + b) * heads + h) * t + query; }
};

// Which particle, sequence, key head, tile and part a workgroup has.  Workgroups go round the eight dies in turn; a die gets ones that
// follow one another.  Four heads, whose keys meet in its L2, take turns tile by tile, so that of causal ones the longest of four heads
// come first and the shortest last: head after head the last head's longest would be left over at the end.  Where a die has less than four
// heads of its own, all heads take turns: otherwise one die would get a head's long tiles and another its short ones (4 x 2 x 2,000 x 8
// heads over 2 of 64 fp16, causal, with documents: forward 89 us, so 68, both with two blocks to a wave; 2 x 2,048 x 8 heads of 64 bf16,
// causal, queries in two parts 38.5, so 32.4).
struct AttnBlock {
    static constexpr int kHeads = 4;
    int particle, batch, head, tile, part;
    bool any;
    __device__ __forceinline__ AttnBlock(const AttnArgs &a)
    {
        const int each = a.tiles * a.splits, heads = a.n * a.batch * a.kv;
        const bool few = heads < 8 * kHeads;
        const int id = few ? (int)blockIdx.x : (int)(blockIdx.x & 7) * a.per_die + (int)(blockIdx.x >> 3);
        any = id < a.total;
        const int in_turn = few ? heads : kHeads, group = id / (in_turn * each), left = id - group * (in_turn * each);
        const int of = max(min(in_turn, heads - group * in_turn), 1); // (the last heads may be fewer; beyond the last one it does not matter)
        const int turn = left / of;
        int h = group * in_turn + left - turn * of;
        tile = turn / a.splits;
        part = turn - tile * a.splits;
        head = h % a.kv;
        h /= a.kv;
        batch = h % a.batch;
        particle = h / a.batch;
    }
};

// ---------------------------------------------------------------------------------------------
// operands
// ---------------------------------------------------------------------------------------------
// Eight values of k of one row, lane l: row l % 16, group l / 16 of k.  16-bit values are as they are; fp32 ones three bf16 parts whose sum
// is the value exactly (split3): the products of parts that are not below 2^-24 of the whole, six, take 96 cycles of a matrix core for 32
// values of k, where the fp32 matrix instructions take 256.
template <class T> struct FragOf {
    typedef T type __attribute__((ext_vector_type(8)));
};
template <> struct FragOf<float> {
    typedef Split3 type;
};
template <class T> using Frag = typename FragOf<T>::type;
template <class T> constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;

__device__ __forceinline__ f32x4 mma(Frag<bf16_t> a, Frag<bf16_t> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(Frag<f16_t> a, Frag<f16_t> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(const Split3 &a, const Split3 &b, f32x4 c)
{
    c = mma(a.l, b.h, c);
    c = mma(a.m, b.m, c);
    c = mma(a.h, b.l, c);
    c = mma(a.m, b.h, c);
    c = mma(a.h, b.m, c);
    return mma(a.h, b.h, c);
}

template <class T> __device__ __forceinline__ float value_of(const Frag<T> &f, int e)
{
    if constexpr (sizeof(T) == 4) return (float)f.h[e] + ((float)f.m[e] + (float)f.l[e]);
    else return (float)f[e];
}

// Heads of less than eight values have kernels of their own, numbered 0: blocks of 32 values, loaded one by one.
template <int KDX> constexpr int kBlocks32 = KDX ? KDX : 1;

// Eight values from memory, those from `left` on 0 and not read.
template <class T> __device__ __forceinline__ Frag<T> load_frag(const T *p, int left, const SplitConst &sc)
{
    typename Pack<T, 8>::raw v;
    if (left >= 8) {
        v = *reinterpret_cast<const typename Pack<T, 8>::type *>(p);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = (T)0.f;
            if (e < left) v[e] = p[e];
        }
    }
    if constexpr (sizeof(T) == 4) return split3(f32x4{v[0], v[1], v[2], v[3]}, f32x4{v[4], v[5], v[6], v[7]}, sc);
    else return v;
}

// ROWS rows of up to 32 KD values in LDS, eight values at a time, brought by THREADS threads, neighbours in the workgroup; of fp32 values
// three planes of parts, made on the way.  Which place of its row such a piece takes is permuted so that what is read at a time meets in no
// bank, of which there are 64: 32 bytes of eight rows in succession (`columns`, by 32 lanes), and of `rows` not one piece of 16 rows but,
// since the lanes 0 .. 3, 12 .. 15 and 20 .. 27 read 16 bytes each together and those between them, a piece of eight rows and the next one
// of the eight others (SQ_LDS_BANK_CONFLICT 0 for either and for the stores; as though lanes 0 .. 15 read together, half the cycles of
// `rows`).  TINY: heads of less than eight values.
template <class T, int KD, bool TINY, int ROWS, int THREADS> struct Tile {
    typedef typename std::conditional<sizeof(T) == 4, bf16_t, T>::type elem; // in LDS
    static constexpr int VEC = 8, kRows = ROWS, kChunks = 32 * KD / VEC, kPlane = ROWS * 32 * KD, kSize = kPlanes<T> * kPlane, N = ROWS * kChunks / THREADS;
    static_assert(N * THREADS == ROWS * kChunks, "every thread has as many pieces");
    typedef typename Pack<T, VEC>::raw raw;
    raw v[N];
    static __device__ __forceinline__ int place(int row, int chunk) // in eight values; moves with the row by 16
    {
        int f;
        if constexpr (KD == 4) f = (row & 7) << 1;
        else if constexpr (KD == 2) f = ((row >> 1) & 3) << 1;
        else f = ((row >> 2) & 1) << 1;
        return row * kChunks + (chunk ^ f);
    }
    static __device__ __forceinline__ int row_of(int u) { return ((int)(threadIdx.x & (THREADS - 1)) + THREADS * u) / kChunks; }
    static __device__ __forceinline__ int chunk_of(int u) { return ((int)(threadIdx.x & (THREADS - 1)) + THREADS * u) % kChunks; }
    // Where the thread's pieces lie, in bytes from the tile's first row; row(i): where row i starts, in elements.  A piece that ends beyond
    // the head is loaded further left (and moved to its place by `store`).
    static __device__ __forceinline__ uint32_t column(int u, int dim)
    {
        const int c = chunk_of(u) * VEC;
        return (uint32_t)(TINY || c + VEC <= dim ? c : dim - VEC) * (uint32_t)sizeof(T);
    }
    template <class F> static __device__ __forceinline__ void offsets(uint32_t (&at)[N], int dim, F row)
    {
#pragma unroll
        for (int u = 0; u < N; ++u) at[u] = (uint32_t)row(row_of(u)) * (uint32_t)sizeof(T) + column(u, dim);
    }
    // The same rows `stride` apart, of which those beyond `last` are not there: that one again.
    __device__ __forceinline__ void load(const T *base, const uint32_t (&at)[N], uint32_t stride, int last, int dim)
    {
        uint32_t to[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const uint32_t most = (uint32_t)last * stride * (uint32_t)sizeof(T) + column(u, dim);
            to[u] = at[u] < most ? at[u] : most;
        }
        load(base, to, dim);
    }
    // Without a branch, so that nothing waits for what is on its way.
    __device__ __forceinline__ void load(const T *base, const uint32_t (&at)[N], int dim)
    {
        const char *const from = reinterpret_cast<const char *>(base);
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if constexpr (TINY) {
                const int c = chunk_of(u) * VEC;
                const T *const p = reinterpret_cast<const T *>(from + (at[u] - column(u, dim)));
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[u][e] = p[c + e < dim ? c + e : dim - 1];
            } else {
                // (a wave's own tiles are read once: 8 x 4 sequences of 4,096 to 8,192 keys, 4 heads of 128 bf16 80 us, so as what others
                // read too 92)
                if constexpr (THREADS == 64) v[u] = __builtin_nontemporal_load(reinterpret_cast<const typename Pack<T, VEC>::type *>(from + at[u]));
                else v[u] = *reinterpret_cast<const typename Pack<T, VEC>::type *>(from + at[u]);
            }
        }
    }
    // What is not there becomes 0 on its way.
    __device__ __forceinline__ void store(elem *lds, int count, int dim, const SplitConst &sc)
    {
        if (!TINY && dim % VEC) {
            const int by = VEC - dim % VEC;
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int c = chunk_of(u) * VEC;
                const bool last = c < dim && c + VEC > dim;
#pragma unroll
                for (int step = 1; step < VEC; step *= 2) {
                    if (!(by & step)) continue;
#pragma unroll
                    for (int e = 0; e + step < VEC; ++e) v[u][e] = last ? v[u][e + step] : v[u][e];
                }
            }
        }
        if (count < ROWS || dim < 32 * KD) {
#pragma unroll
            for (int u = 0; u < N; ++u)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (row_of(u) >= count || chunk_of(u) * VEC + e >= dim) v[u][e] = (T)0.f;
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            Frag<elem> *const to = reinterpret_cast<Frag<elem> *>(lds) + place(row_of(u), chunk_of(u));
            if constexpr (sizeof(T) == 4) {
                const Split3 x = split3(f32x4{v[u][0], v[u][1], v[u][2], v[u][3]}, f32x4{v[u][4], v[u][5], v[u][6], v[u][7]}, sc);
                to[0] = x.h;
                to[kPlane / 8] = x.m;
                to[2 * (kPlane / 8)] = x.l;
            } else {
                *to = v[u];
            }
        }
    }
    // Rows whose log is infinite become 0 in LDS.  (The piece's number is hidden from the compiler, which would keep its places in
    // registers all the time.)
    static __device__ __forceinline__ void clear(elem *lds, const float *log)
    {
        int piece = threadIdx.x & (THREADS - 1);
        asm volatile("" : "+v"(piece));
#pragma unroll 1
        for (; piece < ROWS * kChunks; piece += THREADS) {
            const int row = piece / kChunks;
            if (log[row] != INFINITY) continue;
            Frag<elem> *const to = reinterpret_cast<Frag<elem> *>(lds) + place(row, piece - row * kChunks);
#pragma unroll
            for (int p = 0; p < kPlanes<T>; ++p) to[p * (kPlane / 8)] = Frag<elem>{};
        }
    }
    // operand of rows row .. row + 15, values col .. col + 31
    static __device__ __forceinline__ Frag<T> rows(const elem *lds, int row, int col)
    {
        const int lane = threadIdx.x & 63;
        const Frag<elem> *const p = reinterpret_cast<const Frag<elem> *>(lds) + row * kChunks + place(lane & 15, col / VEC + (lane >> 4));
        if constexpr (sizeof(T) == 4) return {p[0], p[kPlane / 8], p[2 * (kPlane / 8)]};
        else return *p;
    }
    // operand of values col .. col + 15 (its rows), rows row .. row + 31 (its k, ordered 4 g + 0 .. 3, 16 + 4 g + 0 .. 3)
    static __device__ __forceinline__ Frag<T> columns(const elem *lds, int row, int col)
    {
        const int lane = threadIdx.x & 63, g = lane >> 4;
        // (16 lanes read 4 rows of 16 values, a lane the four values of the rows' column lane % 16)
        const elem *const p = lds + row * 32 * KD + place(4 * g + ((lane & 15) >> 2), col / VEC + ((lane & 3) >> 1)) * VEC + 4 * (lane & 1);
        if constexpr (sizeof(T) == 4) return {turned(p), turned(p + kPlane), turned(p + 2 * kPlane)};
        else return turned(p);
    }
    static __device__ __forceinline__ Frag<elem> turned(const elem *p)
    {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds16x4;
        typedef elem t4 __attribute__((ext_vector_type(4)));
        const t4 lo = __builtin_bit_cast(t4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16x4 *)p));
        const t4 hi = __builtin_bit_cast(t4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16x4 *)(p + 16 * 32 * KD)));
        return Frag<elem>{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    }
};

// Streamed tiles of a workgroup: 64 rows, in two halves of LDS, of which one is worked on while the other is filled.  fp32 ones take half
// as much more than the values: 32 rows, or one half alone, so that two or three workgroups fit a CU.
template <class T, int KD> constexpr int kStreamed = sizeof(T) == 4 && KD % 2 == 0 ? 32 : kTileRows;
template <class T, int KD> constexpr int kHalves = sizeof(T) == 4 && KD > 2 ? 1 : 2;
template <class T, int KD, bool TINY> using Streamed = Tile<T, KD, TINY, kStreamed<T, KD>, kAttnBlock>;

// Waits for the loads so far.  Before the loop over tiles: the compiler, which cannot tell an operand loaded before it from a tile loaded
// in it, would wait for the next tile with every tile.
__device__ __forceinline__ void loads_done() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// The part's share of the tiles begin .. end - 1.
__device__ __forceinline__ void part_of(const AttnArgs &a, int part, int &begin, int &end)
{
    const int count = end > begin ? end - begin : 0, first = begin;
    begin = first + (int)((int64_t)count * part / a.splits);
    end = first + (int)((int64_t)count * (part + 1) / a.splits);
}

// What the kernels are built for; told so, the compiler keeps products out of the accumulation registers, which cost a move for every value
// (forward, 4 x 2 x 4,096 x 16 heads of 64 bf16, causal: 604 us, so 468).
constexpr int kWavesPerSimd = 2;

// Two results of 16 streamed rows each as a B operand.
template <class T> __device__ __forceinline__ Frag<T> as_operand(f32x4 a, f32x4 b, const SplitConst &sc)
{
    if constexpr (sizeof(T) == 4) {
        return split3(a, b, sc);
    } else {
        Frag<T> f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[e] = (T)a[e];
            f[4 + e] = (T)b[e];
        }
        return f;
    }
}

// The same in two parts whose sum is the value but for 2^-17 (bf16) or 2^-22 (fp16) of it, which is little beside the 2^-9 or 2^-12 that an
// output's own rounding takes: how probabilities and the gradients of scores become operands.  fp32 is one operand.
template <class T> constexpr int kOperands = 2;
template <> inline constexpr int kOperands<float> = 1;
template <class T> __device__ __forceinline__ void as_parts(f32x4 a, f32x4 b, const SplitConst &sc, Frag<T> (&out)[kOperands<T>])
{
    out[0] = as_operand<T>(a, b, sc);
    if constexpr (std::is_same<T, bf16_t>::value) { // (what is left of a pair: one dot product each, see split3)
        const bf16x2 neg_lo = __builtin_bit_cast(bf16x2, sc.neg_lo), neg_hi = __builtin_bit_cast(bf16x2, sc.neg_hi);
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
            const bf16x2 p = {out[0][k], out[0][k + 1]}, q = {out[0][4 + k], out[0][5 + k]};
            a[k] = __builtin_amdgcn_fdot2_f32_bf16(p, neg_lo, a[k], false);
            a[k + 1] = __builtin_amdgcn_fdot2_f32_bf16(p, neg_hi, a[k + 1], false);
            b[k] = __builtin_amdgcn_fdot2_f32_bf16(q, neg_lo, b[k], false);
            b[k + 1] = __builtin_amdgcn_fdot2_f32_bf16(q, neg_hi, b[k + 1], false);
        }
        out[1] = as_operand<T>(a, b, sc);
    } else if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            a[e] -= (float)out[0][e];
            b[e] -= (float)out[0][4 + e];
        }
        out[1] = as_operand<T>(a, b, sc);
    }
}

// The largest of the four lanes l, l ^ 16, l ^ 32, l ^ 48, in all of them.
__device__ __forceinline__ float max_over_rows(float v)
{
    const unsigned u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const float s = __builtin_elementwise_maximum(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const unsigned w = __float_as_uint(s);
    const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return __builtin_elementwise_maximum(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// The largest of the 16 lanes of a row, in all of them (as row_sum goes).
__device__ __forceinline__ float row_max(float v)
{
    v = __builtin_elementwise_maximum(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xF, 0xF, false)));
    v = __builtin_elementwise_maximum(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xF, 0xF, false)));
    v = __builtin_elementwise_maximum(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xF, 0xF, false)));
    return __builtin_elementwise_maximum(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xF, 0xF, false)));
}

// tanh, for 16-bit activations: up to 1/2 x times a polynomial in x^2 (through its values at the nodes of Chebyshev; off by 1.4e-8, rounded
// by 1.2e-7 of itself), beyond from one exponential, off by 2^-23 or so of 1, which of a small one would be too much: the cap times that is
// the error of an exponent.  For fp32 the library's.
constexpr float kTanhSmall = 0.5f;
__device__ __forceinline__ float tanh_small(float x)
{
    const float u = x * x;
    return x * __builtin_fmaf(u, __builtin_fmaf(u, __builtin_fmaf(u, __builtin_fmaf(u, 0.01714132f, -0.05298924f), 0.13324828f), -0.3333307f), 1.f);
}
__device__ __forceinline__ float tanh_any(float x)
{
    const float large = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * (2.f * kLog2e)));
    return fabsf(x) <= kTanhSmall ? tanh_small(x) : large;
}

// Scores that are capped, or less a slope times the distance: z = out t - slope distance in exponents of 2, where t = tanh(scale s / cap)
// and out = cap, or t = scale s and out = 1; d z / d (scale s) is 1 - on t^2, on = 1 or 0.
struct Modified {
    float in, out, on;
    __device__ __forceinline__ Modified(const AttnArgs &a) : in(a.cap > 0.f ? a.scale / a.cap : a.scale), out((a.cap > 0.f ? a.cap : 1.f) * kLog2e), on(a.cap > 0.f ? 1.f : 0.f) {}
    // s becomes t
    template <class T, int N, int B> __device__ __forceinline__ void apply(f32x4 (&s)[N][B]) const
    {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int b = 0; b < B; ++b) s[j][b] *= in;
        if (on == 0.f) return;
        bool small = sizeof(T) == 2;
        if constexpr (sizeof(T) == 2) {
            float most = 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int b = 0; b < B; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) most = fmaxf(most, fabsf(s[j][b][e]));
            small = __ballot(most > kTanhSmall) == 0; // (mostly)
        }
        if (small) {
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int b = 0; b < B; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[j][b][e] = tanh_small(s[j][b][e]);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int b = 0; b < B; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[j][b][e] = sizeof(T) == 4 ? tanhf(s[j][b][e]) : tanh_any(s[j][b][e]);
        }
    }
    __device__ __forceinline__ float exponent(float t, float slope, float distance) const { return __builtin_fmaf(t, out, -slope * distance); } // slope: times log2 e
    __device__ __forceinline__ float damp(float t) const { return __builtin_fmaf(-on * t, t, 1.f); }
};

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

// Narrows the streamed places [lo, hi) to those from the first to the last that may share a document with one of the places [first, last]:
// all threads of the workgroup call it.
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

// fp16 operands made of sums' terms (dz): scaled by a power of two that keeps the largest so far below 2^15, by wave.  Without it gradients
// below 6e-5 would lose their digits and those beyond 65,504 be infinite.
struct BlockScale {
    float scale = 0x1p100f;
    // the factor by which what was summed up so far has to be multiplied (mostly 1), given the lane's largest new magnitude
    __device__ __forceinline__ float take(float largest)
    {
        largest = row_max(largest);
        largest = max_over_rows(largest);
        if (!(largest * scale > 32768.f)) return 1.f;
        const float next = ldexpf(1.f, min(max(14 - __builtin_amdgcn_frexp_expf(largest), -126), 100));
        const float factor = next / scale;
        scale = next;
        return factor;
    }
};

} // namespace svgd
