// Attention, forward.  A workgroup has 64 QB rows, a wave 16 QB of them; tiles of 64 keys and their values go through two halves of LDS,
// the next tile being on its way from memory while one is worked on.  One pass with the running maximum and sum: sums are rescaled only
// where a maximum rises by more than 2^8. 4 x 2 x 4,096 x 16 heads of 64 bf16, causal: 466 us, 885 TFLOP/s of the three products made (590
// of the two of the formula).  Exponentials, maxima and sums take as long as the products and run beside them only in part: a matrix
// instruction keeps the vector ALU of its SIMD for some 40 % of its time.  8 x 8 x 197 x 6 heads of 64 bf16: 20 us, four tiles a workgroup.
#pragma once
#include "attention_common.hpp"

namespace svgd {

// Probabilities, relative to the running maximum, go into their product with the values in two parts of the activations' type (as_parts):
// in one, half a step off each, with signs as random as those of o's own rounding, they would put o off by 1.1 to 1.4 times what rounding
// it does.  The third product takes 4 x 2 x 4,096 x 16 heads of 64 bf16, causal, from 360 to 466 us, a cache's tokens nothing.  fp16 ones
// are held 2^6 times as large, so that those down to 2^-20 keep their digits.
template <class T> constexpr float kProbExponent = 0.f;
template <> inline constexpr float kProbExponent<f16_t> = 6.f;

// Running maxima and sums of a wave's rows, and their sums of values, of which value 16 d + 4 (lane / 16) + e of row lane % 16 is
// acc[d][b][e].
template <class T, int KD, int QB> struct Running {
    f32x4 acc[2 * KD][QB];
    float top[QB], total[QB]; // total: of the lane's keys
    __device__ __forceinline__ Running()
    {
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            top[b] = -INFINITY;
            total[b] = 0.f;
#pragma unroll
            for (int d = 0; d < 2 * KD; ++d) acc[d][b] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    // Probabilities, relative to the maximum, of NB blocks of 16 keys from their scores, which times mul are exponents of 2.
    template <int NB> __device__ __forceinline__ void probabilities(f32x4 (&s)[NB][QB], float mul, Frag<T> (&p)[NB / 2][QB][kOperands<T>], const SplitConst &sc)
    {
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            float most = s[0][b][0]; // (maximum needs no step that makes signalling NaN quiet first, as fmaxf does)
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) most = __builtin_elementwise_maximum(most, s[j][b][e]);
            most = max_over_rows(most);
            if (__any(most * mul > top[b] * mul + 8.f)) {
                const float next = fmaxf(top[b], most);
                const float factor = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((top[b] - next) * mul);
                top[b] = next;
                total[b] *= factor;
#pragma unroll
                for (int d = 0; d < 2 * KD; ++d) acc[d][b] *= factor;
            }
            const float base = top[b] == -INFINITY ? 0.f : kProbExponent<T> - top[b] * mul;
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[j][b][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j][b][e], mul, base));
                    total[b] += s[j][b][e];
                }
#pragma unroll
            for (int j = 0; j < NB / 2; ++j) as_parts<T>(s[2 * j][b], s[2 * j + 1][b], sc, p[j][b]);
        }
    }
};

template <class T, int KDX, int QB, bool MOD>
__global__ __launch_bounds__(kAttnBlock) __attribute__((amdgpu_waves_per_eu(kWavesPerSimd))) void attention_forward_kernel(AttnArgs a, Heads<const T> q, Heads<const T> k, Heads<const T> v, Heads<T> o,
                                                                                                              float *lse, float *partial, float *partial_lse)
{
    constexpr int KD = kBlocks32<KDX>;
    typedef Streamed<T, KD, KDX == 0> TL;
    constexpr int kRows = TL::kRows, kBuffers = kHalves<T, KD>;
    __shared__ __attribute__((aligned(16))) typename TL::elem lds[2 * kBuffers * TL::kSize];
    __shared__ int red[4], key_documents[kBuffers][kRows];
    const AttnBlock at(a);
    if (!at.any) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    const int tile = a.causal ? a.tiles - 1 - at.tile : at.tile; // (those with the most keys first)
    const int first = tile * (16 * QB * kAttnWaves), own = first + wave * 16 * QB;
    const Masks masks(a, at.batch);
    const float mul = MOD ? 1.f : a.scale * kLog2e; // scores times this are exponents of 2
    const Modified modified(a);
    const SplitConst sc = split_const();

    Frag<T> qf[QB][KD];
    int limit[QB], position[QB], document[QB];
    float slope[QB];
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int r = min(own + 16 * b + (lane & 15), a.rows - 1), i = a.query(r), h = r - i * a.group;
        const T *const p = q.at(at.particle, at.batch, at.head * a.group + h) + i * q.token;
#pragma unroll
        for (int s = 0; s < KD; ++s) qf[b][s] = load_frag(p + 32 * s + 8 * g, a.dim - 32 * s - 8 * g, sc);
        position[b] = masks.start + i;
        limit[b] = masks.end(a, position[b]);
        document[b] = masks.document(a, position[b]);
        slope[b] = MOD && a.slopes ? a.slopes[at.particle * a.slopes_stride + at.head * a.group + h] * kLog2e : 0.f;
    }
    // the keys that the workgroup needs, and up to which a tile needs no mask
    const int last_row = min(first + 16 * QB * kAttnWaves, a.rows) - 1;
    const int p0 = masks.start + a.query(first), p1 = masks.start + a.query(last_row);
    int lo = 0, hi = masks.documents ? (p1 < 0 || p0 >= a.s ? 0 : masks.end(a, min(p1, a.s - 1))) : masks.end(a, p1);
    const int free_keys = masks.documents ? 0 : masks.end(a, p0); // (positions rise with the rows)
    if (masks.documents) narrow(masks.documents, p0, p1, a.s, red, lo, hi);
    int begin = lo / kRows, end = (hi + kRows - 1) / kRows;
    part_of(a, at.part, begin, end);
    const int wave_row = min(own + 16 * QB, a.rows) - 1;
    const int wave_limit = own >= a.rows ? 0 : masks.documents ? hi : masks.end(a, masks.start + a.query(wave_row));

    Running<T, KD, QB> run;
    const T *const ks = k.at(at.particle, at.batch, at.head), *const vs = v.at(at.particle, at.batch, at.head);
    TL kt, vt;
    uint32_t k_at[TL::N], v_at[TL::N];
    TL::offsets(k_at, a.dim, [&](int i) { return (uint32_t)i * (uint32_t)k.token; });
    TL::offsets(v_at, a.dim, [&](int i) { return (uint32_t)i * (uint32_t)v.token; });
    int next_document = 0;
    const auto fetch = [&](int tile_of) {
        const int key = tile_of * kRows, last = min(hi - key, kRows) - 1;
        kt.load(ks + key * k.token, k_at, (uint32_t)k.token, last, a.dim);
        vt.load(vs + key * v.token, v_at, (uint32_t)v.token, last, a.dim);
        if (masks.documents && threadIdx.x < kRows) next_document = key + (int)threadIdx.x < a.s ? masks.documents[key + threadIdx.x] : 0;
    };
    const auto stage = [&](int half, int tile_of) {
        kt.store(lds + half * 2 * TL::kSize, hi - tile_of * kRows, a.dim, sc);
        vt.store(lds + (half * 2 + 1) * TL::kSize, hi - tile_of * kRows, a.dim, sc);
        if (masks.documents && threadIdx.x < kRows) key_documents[half][threadIdx.x] = next_document;
    };
    if (begin < end) {
        fetch(begin);
        stage(0, begin);
    }
    loads_done();
    __syncthreads();
    int half = 0;
    for (int n = begin; n < end; ++n) {
        if (n + 1 < end) fetch(n + 1);
        const int key = n * kRows;
        if (key < wave_limit) {
            const typename TL::elem *const kl = lds + half * 2 * TL::kSize, *const vl = kl + TL::kSize;
            f32x4 s[kRows / 16][QB];
#pragma unroll
            for (int j = 0; j < kRows / 16; ++j) {
#pragma unroll
                for (int b = 0; b < QB; ++b) s[j][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < KD; ++c) {
                    const Frag<T> f = TL::rows(kl, 16 * j, 32 * c);
#pragma unroll
                    for (int b = 0; b < QB; ++b) s[j][b] = mma(f, qf[b][c], s[j][b]);
                }
            }
            if constexpr (MOD) {
                modified.template apply<T>(s);
                if (a.slopes) {
#pragma unroll
                    for (int j = 0; j < kRows / 16; ++j)
#pragma unroll
                        for (int b = 0; b < QB; ++b)
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[j][b][e] = modified.exponent(s[j][b][e], slope[b], fabsf((float)(position[b] - (key + 16 * j + 4 * g + e))));
                } else {
#pragma unroll
                    for (int j = 0; j < kRows / 16; ++j)
#pragma unroll
                        for (int b = 0; b < QB; ++b) s[j][b] *= modified.out;
                }
            }
            if (key + kRows > free_keys) {
#pragma unroll
                for (int j = 0; j < kRows / 16; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int at_key = key + 16 * j + 4 * g + e;
                        const int doc = masks.documents ? key_documents[half][16 * j + 4 * g + e] : 0;
#pragma unroll
                        for (int b = 0; b < QB; ++b)
                            if (at_key >= limit[b] || doc != document[b]) s[j][b][e] = -INFINITY;
                    }
            }
            Frag<T> p[kRows / 32][QB][kOperands<T>];
            run.probabilities(s, mul, p, sc);
#pragma unroll
            for (int j = 0; j < kRows / 32; ++j)
#pragma unroll
                for (int d = 0; d < 2 * KD; ++d) {
                    const Frag<T> f = TL::columns(vl, 32 * j, 16 * d);
#pragma unroll
                    for (int part = 0; part < kOperands<T>; ++part)
#pragma unroll
                        for (int b = 0; b < QB; ++b) run.acc[d][b] = mma(f, p[j][b][part], run.acc[d][b]);
                }
        }
        if constexpr (kBuffers == 2) half ^= 1;
        else __syncthreads(); // (the tile has been read)
        if (n + 1 < end) stage(half, n + 1);
        __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int r = own + 16 * b + (lane & 15);
        const float sum = sum_over_rows(run.total[b]);
        if (r >= a.rows) continue;
        const bool none = sum == 0.f;
        const float inverse = none ? 0.f : 1.f / sum;
        const float log = none ? -INFINITY : (run.top[b] * mul - kProbExponent<T> + __builtin_amdgcn_logf(sum)) * kLn2;
        const int i = a.query(r), h = at.head * a.group + r - i * a.group;
        const int64_t line = a.line(at.particle, at.batch, h, i), lines = (int64_t)a.n * a.batch * a.heads * a.t;
        if (a.splits > 1) {
            if (g == 0) partial_lse[at.part * lines + line] = log;
            float *const out = partial + (at.part * lines + line) * (32 * KD);
#pragma unroll
            for (int d = 0; d < 2 * KD; ++d) *reinterpret_cast<f32x4 *>(out + 16 * d + 4 * g) = none ? f32x4{0.f, 0.f, 0.f, 0.f} : run.acc[d][b] * inverse;
        } else {
            if (g == 0 && lse) lse[line] = log;
            T *const out = o.at(at.particle, at.batch, h) + i * o.token;
#pragma unroll
            for (int d = 0; d < 2 * KD; ++d) {
                const int c = 16 * d + 4 * g;
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = none ? 0.f : run.acc[d][b][e] * inverse;
                if (c < a.dim) store_pack<T, 4>(out + c, a.dim - c, x);
            }
        }
    }
}

// Up to 16 rows: single tokens, or a few, over a cache.  All four waves have the same rows; each takes every fourth tile of 32 keys through
// a part of LDS of its own, so that none waits for another before the end, when their sums are joined.  Reading keys and values once bounds
// it: 8 x 4 x 1 over up to 8,192 x 4 heads of 128 bf16, 486 MB, 79 us, 6.1 TB/s, and the join of 8 parts 4.6; 16 x 1 over 200 x 4 heads of
// 64 fp32 10 us, the chain of one load, two products and the join, twice.
constexpr int kFewKeys = 32;
template <class T, int KDX, bool MOD>
__global__ __launch_bounds__(kAttnBlock) void attention_few_kernel(AttnArgs a, Heads<const T> q, Heads<const T> k, Heads<const T> v, Heads<T> o, float *lse, float *partial, float *partial_lse)
{
    constexpr int KD = kBlocks32<KDX>;
    typedef Tile<T, KD, KDX == 0, kFewKeys, 64> TL;
    constexpr int kJoin = 16 * (32 * KD + 4); // floats of a wave's sums: rows four floats apart from what would be one bank
    constexpr bool kOne = sizeof(T) == 4 && KD > 2; // values where the keys were, once these are read: both do not fit
    constexpr int kTiles = (kOne ? 1 : 2) * TL::kSize * 2, kPart = kTiles > kJoin * 4 ? kTiles : kJoin * 4;
    __shared__ __attribute__((aligned(16))) char lds[kAttnWaves][kPart];
    __shared__ float tops[kAttnWaves][16], totals[kAttnWaves][16];
    const AttnBlock at(a);
    if (!at.any) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    const Masks masks(a, at.batch);
    const float mul = MOD ? 1.f : a.scale * kLog2e;
    const Modified modified(a);
    const SplitConst sc = split_const();
    const int r = min(lane & 15, a.rows - 1), i = a.query(r), h = at.head * a.group + r - i * a.group;
    const T *const qp = q.at(at.particle, at.batch, h) + i * q.token;
    Frag<T> qf[1][KD];
#pragma unroll
    for (int s = 0; s < KD; ++s) qf[0][s] = load_frag(qp + 32 * s + 8 * g, a.dim - 32 * s - 8 * g, sc);
    const int position = masks.start + i, limit = masks.end(a, position), document = masks.document(a, position);
    const float slope = MOD && a.slopes ? a.slopes[at.particle * a.slopes_stride + h] * kLog2e : 0.f;
    const int p0 = masks.start, p1 = masks.start + a.t - 1;
    const int hi = masks.documents ? (p1 < 0 || p0 >= a.s ? 0 : masks.end(a, min(p1, a.s - 1))) : masks.end(a, p1);
    const int free_keys = masks.documents ? 0 : masks.end(a, p0);
    int begin = 0, end = (hi + kFewKeys - 1) / kFewKeys;
    part_of(a, at.part, begin, end);

    Running<T, KD, 1> run;
    const T *const ks = k.at(at.particle, at.batch, at.head), *const vs = v.at(at.particle, at.batch, at.head);
    typename TL::elem *const kl = reinterpret_cast<typename TL::elem *>(lds[wave]), *const vl = kOne ? kl : kl + TL::kSize;
    TL kt, vt;
    uint32_t k_at[TL::N], v_at[TL::N];
    TL::offsets(k_at, a.dim, [&](int j) { return (uint32_t)j * (uint32_t)k.token; });
    TL::offsets(v_at, a.dim, [&](int j) { return (uint32_t)j * (uint32_t)v.token; });
    const auto fetch = [&](int n) {
        const int key = n * kFewKeys, last = min(hi - key, kFewKeys) - 1;
        kt.load(ks + key * k.token, k_at, (uint32_t)k.token, last, a.dim);
        vt.load(vs + key * v.token, v_at, (uint32_t)v.token, last, a.dim);
    };
    loads_done();
    if (begin + wave < end) fetch(begin + wave);
    for (int n = begin + wave; n < end; n += kAttnWaves) {
        const int key = n * kFewKeys;
        wave_sync(); // (the tile before has been read)
        kt.store(kl, hi - key, a.dim, sc);
        if constexpr (!kOne) vt.store(vl, hi - key, a.dim, sc);
        wave_sync();
        if constexpr (!kOne)
            if (n + kAttnWaves < end) fetch(n + kAttnWaves);
        f32x4 s[2][1];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            s[j][0] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < KD; ++c) s[j][0] = mma(TL::rows(kl, 16 * j, 32 * c), qf[0][c], s[j][0]);
        }
        if constexpr (kOne) {
            wave_sync();
            vt.store(vl, hi - key, a.dim, sc);
            wave_sync();
            if (n + kAttnWaves < end) fetch(n + kAttnWaves);
        }
        if constexpr (MOD) {
            modified.template apply<T>(s);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[j][0][e] = modified.exponent(s[j][0][e], slope, fabsf((float)(position - (key + 16 * j + 4 * g + e))));
        }
        if (key + kFewKeys > free_keys) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at_key = key + 16 * j + 4 * g + e;
                    const int doc = masks.documents ? masks.documents[min(at_key, a.s - 1)] : 0;
                    if (at_key >= limit || doc != document) s[j][0][e] = -INFINITY;
                }
        }
        Frag<T> p[1][1][kOperands<T>];
        run.probabilities(s, mul, p, sc);
#pragma unroll
        for (int d = 0; d < 2 * KD; ++d) {
            const Frag<T> f = TL::columns(vl, 0, 16 * d);
#pragma unroll
            for (int part = 0; part < kOperands<T>; ++part) run.acc[d][0] = mma(f, p[0][0][part], run.acc[d][0]);
        }
    }
    // the waves' sums, in their order
    run.total[0] = sum_over_rows(run.total[0]);
    wave_sync();
    float *const mine = reinterpret_cast<float *>(lds[wave]);
    if (g == 0) {
        tops[wave][lane] = run.top[0];
        totals[wave][lane] = run.total[0];
    }
#pragma unroll
    for (int d = 0; d < 2 * KD; ++d) *reinterpret_cast<f32x4 *>(mine + (lane & 15) * (32 * KD + 4) + 16 * d + 4 * g) = run.acc[d][0];
    __syncthreads();
    for (int x = threadIdx.x; x < a.rows * 8 * KD; x += kAttnBlock) {
        const int row = x / (8 * KD), c = (x - row * 8 * KD) * 4;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) top = __builtin_elementwise_maximum(top, tops[w][row]);
        f32x4 all = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) {
            if (totals[w][row] == 0.f) continue;
            const float share = __builtin_amdgcn_exp2f((tops[w][row] - top) * mul);
            sum += share * totals[w][row];
            all += share * *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(lds[w]) + row * (32 * KD + 4) + c);
        }
        const bool none = sum == 0.f;
        const float inverse = none ? 0.f : 1.f / sum, log = none ? -INFINITY : (top * mul - kProbExponent<T> + __builtin_amdgcn_logf(sum)) * kLn2;
        const int query = a.query(row), head = at.head * a.group + row - query * a.group;
        const int64_t line = a.line(at.particle, at.batch, head, query), lines = (int64_t)a.n * a.batch * a.heads * a.t;
        if (a.splits > 1) {
            if (c == 0) partial_lse[at.part * lines + line] = log;
            *reinterpret_cast<f32x4 *>(partial + (at.part * lines + line) * (32 * KD) + c) = all * inverse;
        } else {
            if (c == 0 && lse) lse[line] = log;
            const float y[4] = {all[0] * inverse, all[1] * inverse, all[2] * inverse, all[3] * inverse};
            if (c < a.dim) store_pack<T, 4>(o.at(at.particle, at.batch, head) + query * o.token + c, a.dim - c, y);
        }
    }
}

// The parts' results, each weighted by its share of the sum of exponentials: a thread has four values of a row.
template <class T> __global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a, int ld, const float *partial, const float *partial_lse, Heads<T> o, float *lse)
{
    const int64_t lines = (int64_t)a.n * a.batch * a.heads * a.t;
    const int quads = ld / 4;
    const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x, line = k / quads;
    const int c = (int)(k - line * quads) * 4;
    if (line >= lines || c >= a.dim) return;
    // eight parts at a time, so that their loads are on their way together
    constexpr int U = 8;
    float top = -INFINITY, total = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < a.splits; p0 += U) {
        float l[U];
        f32x4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t p = min(p0 + u, a.splits - 1);
            l[u] = partial_lse[p * lines + line];
            x[u] = *reinterpret_cast<const f32x4 *>(partial + (p * lines + line) * ld + c);
        }
        float next = top;
#pragma unroll
        for (int u = 0; u < U; ++u) next = __builtin_elementwise_maximum(next, l[u]);
        const float old = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((top - next) * kLog2e);
        total *= old;
        sum *= old;
        top = next;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p0 + u >= a.splits || l[u] == -INFINITY) continue;
            const float w = __builtin_amdgcn_exp2f((l[u] - top) * kLog2e);
            total += w;
            sum += w * x[u];
        }
    }
    const bool none = total == 0.f;
    const float inverse = none ? 0.f : 1.f / total;
    const int i = (int)(line % a.t);
    const int64_t head = line / a.t;
    const int h = (int)(head % a.heads), b = (int)(head / a.heads % a.batch), particle = (int)(head / a.heads / a.batch);
    const float x[4] = {sum[0] * inverse, sum[1] * inverse, sum[2] * inverse, sum[3] * inverse};
    store_pack<T, 4>(o.at(particle, b, h) + i * o.token + c, a.dim - c, x);
    if (c == 0 && lse) lse[line] = none ? -INFINITY : top + __builtin_amdgcn_logf(total) * kLn2;
}

} // namespace svgd
