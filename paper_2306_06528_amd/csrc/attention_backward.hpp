// Attention, backward, without atomics: one kernel has rows of its own and streams keys and values past them (dq, and the slopes' gradients
// row by row), the other has keys of its own and streams rows past them (dk and dv, summed over the heads that share them).  Both make the
// probabilities again from lse: five products and six of 16-bit activations for the forward pass's three.  4 x 2 x 4,096 x 16 heads of 64
// bf16, causal: 732 us (687 Gflop, 938 TFLOP/s) and 842 us (825 Gflop, 980 TFLOP/s), matrix cores and vector ALU taking turns; 8 x 8 x 197
// x 6 heads of 64 bf16: 28.8 and 33.1, four tiles each.  (With P in one part and delta of o as it is stored 621 and 763, 27.1 and 31.2.)
//     P = exp(z - lse),  dP = do v,  dz = P (dP - delta),  delta = sum_c do_c o_c
// P goes into the product with do, and dz into those with k and q, in two parts of the activations' type (BlockScale: fp16), and delta is
// made free of o's rounding (kRestore): dq, dk and dv are off by 1.00 times what rounding them does, whether a row sees 3 keys or 4,096.  P
// in one part would make that 1.4 for dv, delta of o as it is stored 1.1 to 1.8 for dq and dk, the more the fewer keys count.
#pragma once
#include "attention_common.hpp"

namespace svgd {

// o as it was stored leaves delta off by its roundings: by eps, which of rows that see few keys, or few that count, is not small beside dz
// and does not cancel.  The sum of a row's dz is 0, so made with the delta at hand it is eps, and
//     dz = dz0 - eps P,   dq = scale (sum dz0 damp k - eps sum P damp k)
// The kernel that has queries of its own adds up the two sums beside dq's (a fifth product; P in one part does, eps being 2^-9 of delta),
// and leaves delta + eps for the kernel that has keys of its own.  Not for fp32, whose o is rounded as every sum is.
template <class T> constexpr bool kRestore = sizeof(T) == 2;

// One of two forms of a loop, the same for the whole wave.
template <class F> __device__ __forceinline__ void with_mask(bool masked, F f)
{
    if (masked) f(std::true_type{});
    else f(std::false_type{});
}

// delta of every row, 16 lanes each, where the kernel that has queries of its own, which makes it otherwise, is not wanted: fp32.
template <class T> __global__ __launch_bounds__(256) void attention_delta_kernel(AttnArgs a, Heads<const T> o, Heads<const T> d_o, float *delta)
{
    const int64_t k = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4), lines = (int64_t)a.n * a.batch * a.t * a.heads;
    if (k >= lines) return;
    const int h = (int)(k % a.heads);
    const int64_t token = k / a.heads;
    const int i = (int)(token % a.t), b = (int)(token / a.t % a.batch), particle = (int)(token / a.t / a.batch);
    const int c = 8 * (threadIdx.x & 15);
    const SplitConst sc = split_const();
    const Frag<T> x = load_frag(o.at(particle, b, h) + i * o.token + c, a.dim - c, sc), y = load_frag(d_o.at(particle, b, h) + i * d_o.token + c, a.dim - c, sc);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += value_of<T>(x, e) * value_of<T>(y, e);
    sum = row_sum(sum);
    if ((threadIdx.x & 15) == 0) delta[a.line(particle, b, h, i)] = sum;
}

// (Heads of 33 to 64 values, fp16, capped, take 169 and 170 registers left to themselves, one or two more than leave room for three waves:
// 4 x 2 x 2,000 x 8 heads over 2 of 64, causal, 7 documents, queries 116 us, so 95, keys 124, so 114; fp32 would spill 47: keys of 3 x 2 x
// 333 x 6 heads over 2 of 40 29 us, so 23.)
template <class T, int KDX, int B> constexpr int kWavesBackward = sizeof(T) == 2 && KDX == 2 && B == 1 ? 3 : kWavesPerSimd;

template <class T, int KDX, bool MOD>
__global__ __launch_bounds__(kAttnBlock) __attribute__((amdgpu_waves_per_eu(kWavesBackward<T, KDX, 1>))) void attention_queries_kernel(AttnArgs a, Heads<const T> q, Heads<const T> k, Heads<const T> v, Heads<const T> d_o,
                                                                                                              Heads<const T> o, const float *lse, float *delta, Heads<T> dq, float *slope_rows, float *row_sums, float *partial)
{
    constexpr int QB = 1; // blocks of 16 rows of a wave's own (attention_launch.hpp)
    constexpr int KD = kBlocks32<KDX>;
    typedef Streamed<T, KD, KDX == 0> TL;
    constexpr int kRows = TL::kRows, kBuffers = kHalves<T, KD>;
    __shared__ __attribute__((aligned(16))) typename TL::elem lds[2 * kBuffers * TL::kSize];
    __shared__ int red[4], key_documents[kBuffers][kRows];
    const AttnBlock at(a);
    if (!at.any) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    const int tile = a.causal ? a.tiles - 1 - at.tile : at.tile;
    const int first = tile * (16 * QB * kAttnWaves), own = first + wave * 16 * QB;
    const Masks masks(a, at.batch);
    const float mul = MOD ? 1.f : a.scale * kLog2e;
    const Modified modified(a);
    const SplitConst sc = split_const();

    Frag<T> qf[QB][KD], df[QB][KD];
    int limit[QB], position[QB], document[QB];
    float slope[QB], log[QB];
    f32x4 less[QB];
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int r = min(own + 16 * b + (lane & 15), a.rows - 1), i = a.query(r), h = at.head * a.group + r - i * a.group;
        const T *const p = q.at(at.particle, at.batch, h) + i * q.token, *const d = d_o.at(at.particle, at.batch, h) + i * d_o.token;
#pragma unroll
        for (int s = 0; s < KD; ++s) {
            qf[b][s] = load_frag(p + 32 * s + 8 * g, a.dim - 32 * s - 8 * g, sc);
            df[b][s] = load_frag(d + 32 * s + 8 * g, a.dim - 32 * s - 8 * g, sc);
        }
        position[b] = masks.start + i;
        limit[b] = masks.end(a, position[b]);
        document[b] = masks.document(a, position[b]);
        slope[b] = MOD && a.slopes ? a.slopes[at.particle * a.slopes_stride + h] * kLog2e : 0.f;
        const int64_t line = a.line(at.particle, at.batch, h, i);
        log[b] = lse[line] == -INFINITY ? INFINITY : lse[line] * kLog2e; // (a row that sees nothing: every probability 0)
        const T *const op = o.at(at.particle, at.batch, h) + i * o.token;
        float del = 0.f;
#pragma unroll
        for (int s = 0; s < KD; ++s) {
            const Frag<T> f = load_frag(op + 32 * s + 8 * g, a.dim - 32 * s - 8 * g, sc);
#pragma unroll
            for (int e = 0; e < 8; ++e) del += value_of<T>(f, e) * value_of<T>(df[b][s], e);
        }
        del = sum_over_rows(del);
        less[b] = f32x4{-del, -del, -del, -del};
    }
    const int last_row = min(first + 16 * QB * kAttnWaves, a.rows) - 1;
    const int p0 = masks.start + a.query(first), p1 = masks.start + a.query(last_row);
    int lo = 0, hi = masks.documents ? (p1 < 0 || p0 >= a.s ? 0 : masks.end(a, min(p1, a.s - 1))) : masks.end(a, p1);
    const int free_keys = masks.documents ? 0 : masks.end(a, p0);
    if (masks.documents) narrow(masks.documents, p0, p1, a.s, red, lo, hi);
    int begin = lo / kRows, end = (hi + kRows - 1) / kRows;
    part_of(a, at.part, begin, end);
    const int wave_row = min(own + 16 * QB, a.rows) - 1;
    const int wave_limit = own >= a.rows ? 0 : masks.documents ? hi : masks.end(a, masks.start + a.query(wave_row));

    f32x4 acc[2 * KD][QB], mean[kRestore<T> ? 2 * KD : 1][QB]; // of dz k and of P k
    float sum_dz[QB], sum_dz_far[QB], sum_far[QB]; // of dz, dz distance and P distance
    BlockScale bs;
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        sum_dz[b] = sum_dz_far[b] = sum_far[b] = 0.f;
#pragma unroll
        for (int d = 0; d < 2 * KD; ++d) {
            acc[d][b] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (kRestore<T>) mean[d][b] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
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
        const int key0 = n * kRows;
        if (key0 < wave_limit) {
            const typename TL::elem *const kl = lds + half * 2 * TL::kSize, *const vl = kl + TL::kSize;
#pragma unroll
            for (int m = 0; m < kRows / 32; ++m) {
                const int key = key0 + 32 * m;
                f32x4 s[2][QB], dp[2][QB];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int b = 0; b < QB; ++b) {
                        s[j][b] = f32x4{0.f, 0.f, 0.f, 0.f};
                        dp[j][b] = less[b]; // dP - delta, from the start
                    }
#pragma unroll
                    for (int c = 0; c < KD; ++c) {
                        const Frag<T> f = TL::rows(kl, 32 * m + 16 * j, 32 * c), e = TL::rows(vl, 32 * m + 16 * j, 32 * c);
#pragma unroll
                        for (int b = 0; b < QB; ++b) {
                            s[j][b] = mma(f, qf[b][c], s[j][b]);
                            dp[j][b] = mma(e, df[b][c], dp[j][b]);
                        }
                    }
                }
                if constexpr (MOD) modified.template apply<T>(s);
                float largest = 0.f;
                const auto gradients = [&](auto masked, auto biased) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int at_key = key + 16 * j + 4 * g + e;
                            const int doc = masked && masks.documents ? key_documents[half][32 * m + 16 * j + 4 * g + e] : 0;
#pragma unroll
                            for (int b = 0; b < QB; ++b) {
                                float x = s[j][b][e];
                                [[maybe_unused]] const float far = fabsf((float)(position[b] - at_key)), t = x;
                                if constexpr (MOD) x = biased ? modified.exponent(t, slope[b], far) : t * modified.out;
                                if (masked && (at_key >= limit[b] || doc != document[b])) x = -INFINITY;
                                float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x, mul, -log[b])), dz = p * dp[j][b][e];
                                if (biased || kRestore<T>) sum_dz[b] += dz;
                                if (biased) {
                                    sum_dz_far[b] += dz * far;
                                    sum_far[b] += p * far;
                                }
                                if constexpr (MOD) {
                                    const float damp = modified.damp(t);
                                    dz *= damp;
                                    p *= damp;
                                }
                                s[j][b][e] = dz;
                                dp[j][b][e] = p;
                                if constexpr (std::is_same<T, f16_t>::value) largest = fmaxf(largest, fabsf(dz));
                            }
                        }
                };
                const bool some_hidden = key0 + kRows > free_keys;
                if (MOD && a.slopes) with_mask(some_hidden, [&](auto masked) { gradients(masked, std::bool_constant<MOD>{}); });
                else with_mask(some_hidden, [&](auto masked) { gradients(masked, std::false_type{}); });
                if constexpr (std::is_same<T, f16_t>::value) {
                    const float factor = bs.take(largest);
                    if (factor != 1.f) {
#pragma unroll
                        for (int b = 0; b < QB; ++b)
#pragma unroll
                            for (int d = 0; d < 2 * KD; ++d) acc[d][b] *= factor;
                    }
#pragma unroll
                    for (int b = 0; b < QB; ++b) {
                        s[0][b] *= bs.scale;
                        s[1][b] *= bs.scale;
                    }
                }
                Frag<T> z[QB][kOperands<T>], p[QB];
#pragma unroll
                for (int b = 0; b < QB; ++b) {
                    as_parts<T>(s[0][b], s[1][b], sc, z[b]);
                    if constexpr (kRestore<T>) p[b] = as_operand<T>(dp[0][b], dp[1][b], sc);
                }
#pragma unroll
                for (int d = 0; d < 2 * KD; ++d) {
                    const Frag<T> f = TL::columns(kl, 32 * m, 16 * d);
#pragma unroll
                    for (int part = 0; part < kOperands<T>; ++part)
#pragma unroll
                        for (int b = 0; b < QB; ++b) acc[d][b] = mma(f, z[b][part], acc[d][b]);
                    if constexpr (kRestore<T>)
#pragma unroll
                        for (int b = 0; b < QB; ++b) mean[d][b] = mma(f, p[b], mean[d][b]);
                }
            }
        }
        if constexpr (kBuffers == 2) half ^= 1;
        else __syncthreads(); // (the tile has been read)
        if (n + 1 < end) stage(half, n + 1);
        __syncthreads();
    }
    const float factor = std::is_same<T, f16_t>::value ? a.scale / bs.scale : a.scale;
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int r = own + 16 * b + (lane & 15);
        const int i = a.query(min(r, a.rows - 1)), h = at.head * a.group + min(r, a.rows - 1) - i * a.group;
        if (log[b] == INFINITY) { // a row that sees nothing: 0, whatever it holds
            sum_dz[b] = sum_dz_far[b] = sum_far[b] = 0.f;
            less[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int d = 0; d < 2 * KD; ++d) {
                acc[d][b] = f32x4{0.f, 0.f, 0.f, 0.f};
                if constexpr (kRestore<T>) mean[d][b] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
        const int64_t line = a.line(at.particle, at.batch, h, i), lines = (int64_t)a.n * a.batch * a.heads * a.t;
        const float eps = kRestore<T> || MOD ? sum_over_rows(sum_dz[b]) : 0.f;
        if (r < a.rows && g == 0) {
            if (at.part == 0) delta[line] = kRestore<T> && a.splits == 1 ? eps - less[b][0] : -less[b][0];
            if ((kRestore<T> || MOD) && a.splits > 1) row_sums[at.part * lines + line] = eps;
        }
        if constexpr (MOD) {
            // What delta's error puts on the sum with the distances is taken off, in fp32 too (the probabilities add up to 1)
            const float zf = sum_over_rows(sum_dz_far[b]), f = sum_over_rows(sum_far[b]);
            if (a.slopes && slope_rows && r < a.rows && g == 0) {
                if (a.splits > 1) {
                    row_sums[(a.splits + 2 * at.part) * lines + line] = zf;
                    row_sums[(a.splits + 2 * at.part + 1) * lines + line] = f;
                } else {
                    slope_rows[line] = eps * f - zf;
                }
            }
        }
        if (r >= a.rows || !dq.p) continue;
        if (a.splits > 1) {
            constexpr int kEach = kRestore<T> ? 64 * KD : 32 * KD;
            float *const out = partial + (at.part * lines + line) * kEach;
#pragma unroll
            for (int d = 0; d < 2 * KD; ++d) {
                *reinterpret_cast<f32x4 *>(out + 16 * d + 4 * g) = acc[d][b] * factor;
                if constexpr (kRestore<T>) *reinterpret_cast<f32x4 *>(out + 32 * KD + 16 * d + 4 * g) = mean[d][b] * a.scale;
            }
            continue;
        }
        const float off = eps * a.scale;
        T *const out = dq.at(at.particle, at.batch, h) + i * dq.token;
#pragma unroll
        for (int d = 0; d < 2 * KD; ++d) {
            const int c = 16 * d + 4 * g;
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = acc[d][b][e] * factor;
                if constexpr (kRestore<T>) x[e] = __builtin_fmaf(-off, mean[d][b][e], x[e]);
            }
            if (c < a.dim) store_pack<T, 4>(out + c, a.dim - c, x);
        }
    }
}

// What a streamed row brings besides its values.
struct __attribute__((aligned(16))) RowInfo {
    float log[kTileRows], less[kTileRows], slope[kTileRows];
    int limit[kTileRows], position[kTileRows], document[kTileRows];
};

template <class T, int KDX, int KB, bool MOD>
__global__ __launch_bounds__(kAttnBlock) __attribute__((amdgpu_waves_per_eu(kWavesBackward<T, KDX, KB>))) void attention_keys_kernel(AttnArgs a, Heads<const T> q, Heads<const T> k, Heads<const T> v, Heads<const T> d_o,
                                                                                                           const float *lse, const float *delta, Heads<T> dk, Heads<T> dv, float *partial)
{
    constexpr int KD = kBlocks32<KDX>;
    typedef Streamed<T, KD, KDX == 0> TL;
    constexpr int kRows = TL::kRows, kBuffers = kHalves<T, KD>;
    // Two waves to a SIMD hide little of what a wave waits for: operands are asked for well before their products, where the compiler,
    // short of registers, asks for a few at a time and waits for each (4 x 2 x 4,096 x 16 heads of 64 bf16 causal 915 us, so 875; with one
    // block of keys, three waves, the registers are worth more: 8 x 8 x 197 x 6 heads of 64 35 us, so 43).
    constexpr bool kDeep = sizeof(T) == 2 && (KB == 2 || KD > 2);
    constexpr int kEarly = kDeep ? (KD <= 2 ? 2 * KD : 4) : 0; // transposed operands that are asked for before the exponentials
    constexpr bool kHalf = std::is_same<T, f16_t>::value;
    constexpr float kExponent = kHalf ? 14.f : 0.f; // of probabilities as operands
    __shared__ __attribute__((aligned(16))) typename TL::elem lds[2 * kBuffers * TL::kSize];
    __shared__ RowInfo infos[kBuffers];
    __shared__ int red[4];
    const AttnBlock at(a);
    if (!at.any) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    const int first = at.tile * (16 * KB * kAttnWaves), own = first + wave * 16 * KB;
    const Masks masks(a, at.batch);
    const float mul = MOD ? 1.f : a.scale * kLog2e;
    const Modified modified(a);
    const SplitConst sc = split_const();

    Frag<T> kf[KB][KD], vf[KB][KD];
    int key[KB], document[KB];
#pragma unroll
    for (int b = 0; b < KB; ++b) {
        key[b] = own + 16 * b + (lane & 15);
        const bool there = key[b] < masks.length;
        const T *const kp = k.at(at.particle, at.batch, at.head) + key[b] * k.token, *const vp = v.at(at.particle, at.batch, at.head) + key[b] * v.token;
#pragma unroll
        for (int s = 0; s < KD; ++s) {
            const int left = there ? a.dim - 32 * s - 8 * g : 0;
            kf[b][s] = load_frag(kp + 32 * s + 8 * g, left, sc);
            vf[b][s] = load_frag(vp + 32 * s + 8 * g, left, sc);
        }
        document[b] = masks.documents && there ? masks.documents[key[b]] : 0;
    }
    // the rows that may see the workgroup's keys
    int row_lo = 0, row_hi = first < masks.length ? a.rows : 0;
    const int last_key = min(first + 16 * KB * kAttnWaves, masks.length) - 1;
    if (a.causal && masks.prefix <= first) row_lo = (int)min((int64_t)max(first - masks.start, 0) * a.group, (int64_t)a.rows);
    if (masks.documents && row_hi > 0) {
        int lo = masks.start + row_lo / a.group, hi = masks.start + a.t;
        narrow(masks.documents, first, last_key, a.s, red, lo, hi);
        row_lo = hi > lo ? max(row_lo, (lo - masks.start) * a.group) : 0;
        row_hi = hi > lo ? min(a.rows, (hi - masks.start) * a.group) : 0;
    }
    int begin = row_lo / kRows, end = row_hi > row_lo ? (row_hi + kRows - 1) / kRows : begin;
    part_of(a, at.part, begin, end);
    // tiles from this row on need no mask
    const int wave_last = own + 16 * KB - 1;
    const int free_row = masks.documents || wave_last >= masks.length ? INT32_MAX
                         : !a.causal || masks.prefix > wave_last      ? 0
                                                                      : (int)min((int64_t)max(wave_last - masks.start, 0) * a.group, (int64_t)INT32_MAX);

    f32x4 acc_k[2 * KD][KB], acc_v[2 * KD][KB];
    BlockScale bs;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int d = 0; d < 2 * KD; ++d) acc_k[d][b] = acc_v[d][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    TL qt, dt;
    // (tiles begin with a token's first head where the heads of a group divide 64: then the rows of all tiles lie alike)
    const bool steady = kRows % a.group == 0;
    uint32_t q_at[TL::N], d_at[TL::N];
    const auto place = [&](int j, int64_t token, int64_t head) {
        const int i = a.query(j);
        return (uint32_t)i * (uint32_t)token + (uint32_t)(j - i * a.group) * (uint32_t)head;
    };
    TL::offsets(q_at, a.dim, [&](int j) { return place(j, q.token, q.head); });
    TL::offsets(d_at, a.dim, [&](int j) { return place(j, d_o.token, d_o.head); });
    float next_log = 0.f, next_delta = 0.f, next_slope = 0.f;
    int next_limit = 0, next_position = 0, next_document = 0;
    const auto fetch = [&](int tile_of) {
        const int row = tile_of * kRows;
        const int i0 = a.query(row), h0 = row - i0 * a.group, last = min(a.rows - row, kRows) - 1;
        const T *const qs = q.at(at.particle, at.batch, at.head * a.group) + i0 * q.token, *const ds = d_o.at(at.particle, at.batch, at.head * a.group) + i0 * d_o.token;
        if (steady && last == kRows - 1) {
            qt.load(qs, q_at, a.dim);
            dt.load(ds, d_at, a.dim);
        } else {
            uint32_t to[TL::N];
            const auto row_at = [&](int j, int64_t token, int64_t head) {
                const int r = h0 + min(j, last), i = a.query(r);
                return (uint32_t)i * (uint32_t)token + (uint32_t)(r - i * a.group) * (uint32_t)head;
            };
            TL::offsets(to, a.dim, [&](int j) { return row_at(j, q.token, q.head); });
            qt.load(qs, to, a.dim);
            TL::offsets(to, a.dim, [&](int j) { return row_at(j, d_o.token, d_o.head); });
            dt.load(ds, to, a.dim);
        }
        if (threadIdx.x < kRows) {
            const int r = row + (int)threadIdx.x;
            next_log = INFINITY;
            next_delta = next_slope = 0.f;
            next_limit = next_position = next_document = 0;
            if (r < a.rows) {
                const int i = a.query(r), h = at.head * a.group + r - i * a.group;
                const int64_t line = a.line(at.particle, at.batch, h, i);
                next_log = lse[line] == -INFINITY ? INFINITY : lse[line] * kLog2e; // (a row that sees nothing: every probability 0)
                next_delta = delta[line];
                next_position = masks.start + i;
                next_limit = masks.end(a, next_position);
                next_document = masks.document(a, next_position);
                if (MOD && a.slopes) next_slope = a.slopes[at.particle * a.slopes_stride + h] * kLog2e;
            }
        }
    };
    const auto stage = [&](int half, int tile_of) {
        qt.store(lds + half * 2 * TL::kSize, a.rows - tile_of * kRows, a.dim, sc);
        dt.store(lds + (half * 2 + 1) * TL::kSize, a.rows - tile_of * kRows, a.dim, sc);
        if (threadIdx.x < kRows) {
            RowInfo &info = infos[half];
            info.log[threadIdx.x] = next_log;
            info.less[threadIdx.x] = next_log == INFINITY ? 0.f : -next_delta; // (not where it is loaded, which would wait for it)
            info.slope[threadIdx.x] = next_slope;
            info.limit[threadIdx.x] = next_limit;
            info.position[threadIdx.x] = next_position;
            info.document[threadIdx.x] = next_document;
        }
    };
    // Rows that see nothing are 0 in the products, whatever they hold.
    const auto ready = [&](int half) {
        __syncthreads();
        if (!a.blind()) return;
        TL::clear(lds + half * 2 * TL::kSize, infos[half].log);
        TL::clear(lds + (half * 2 + 1) * TL::kSize, infos[half].log);
        __syncthreads();
    };
    if (begin < end) {
        fetch(begin);
        stage(0, begin);
    }
    loads_done();
    ready(0);
    int half = 0;
    for (int n = begin; n < end; ++n) {
        if (n + 1 < end) fetch(n + 1);
        const typename TL::elem *const ql = lds + half * 2 * TL::kSize, *const dl = ql + TL::kSize;
        const RowInfo &info = infos[half];
        const bool masked = n * kRows < free_row;
        if (own < masks.length)
#pragma unroll
            for (int m = 0; m < kRows / 32; ++m) {
                f32x4 s[2][KB], dp[2][KB];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    Frag<T> f[KD], e[KD];
                    const f32x4 less = *reinterpret_cast<const f32x4 *>(&info.less[32 * m + 16 * j + 4 * g]);
#pragma unroll
                    for (int c = 0; c < KD; ++c) {
                        f[c] = TL::rows(ql, 32 * m + 16 * j, 32 * c);
                        e[c] = TL::rows(dl, 32 * m + 16 * j, 32 * c);
                    }
                    if constexpr (kDeep)
                        if (j == 0 || KD > 2) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int b = 0; b < KB; ++b) {
                        s[j][b] = f32x4{0.f, 0.f, 0.f, 0.f};
                        dp[j][b] = less; // dP - delta, from the start
                    }
#pragma unroll
                    for (int c = 0; c < KD; ++c)
#pragma unroll
                        for (int b = 0; b < KB; ++b) {
                            s[j][b] = mma(f[c], kf[b][c], s[j][b]);
                            dp[j][b] = mma(e[c], vf[b][c], dp[j][b]);
                        }
                }
                Frag<T> dc[kEarly + 1];
#pragma unroll
                for (int d = 0; d < kEarly; ++d) dc[d] = TL::columns(dl, 32 * m, 16 * d);
                if constexpr (kDeep) __builtin_amdgcn_sched_barrier(0);
                if constexpr (MOD) modified.template apply<T>(s);
                float largest = 0.f;
                const auto gradients = [&](auto hidden, auto biased) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int r = 32 * m + 16 * j + 4 * g;
                        const f32x4 log = *reinterpret_cast<const f32x4 *>(&info.log[r]);
                        [[maybe_unused]] const f32x4 slope = *reinterpret_cast<const f32x4 *>(&info.slope[r]);
                        [[maybe_unused]] const i32x4 limit = *reinterpret_cast<const i32x4 *>(&info.limit[r]), position = *reinterpret_cast<const i32x4 *>(&info.position[r]),
                                                     documents = *reinterpret_cast<const i32x4 *>(&info.document[r]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
#pragma unroll
                            for (int b = 0; b < KB; ++b) {
                                float x = s[j][b][e];
                                [[maybe_unused]] const float t = x;
                                if constexpr (MOD) x = biased ? modified.exponent(t, slope[e], fabsf((float)(position[e] - key[b]))) : t * modified.out;
                                if (hidden && (key[b] >= limit[e] || document[b] != documents[e])) x = -INFINITY;
                                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x, mul, kExponent - log[e]));
                                float dz = p * dp[j][b][e];
                                if constexpr (MOD) dz *= modified.damp(t);
                                s[j][b][e] = p;
                                dp[j][b][e] = dz;
                                if constexpr (kHalf) largest = fmaxf(largest, fabsf(dz));
                            }
                        }
                    }
                };
                if (MOD && a.slopes) with_mask(masked, [&](auto hidden) { gradients(hidden, std::bool_constant<MOD>{}); });
                else with_mask(masked, [&](auto hidden) { gradients(hidden, std::false_type{}); });
                if constexpr (kHalf) {
                    const float factor = bs.take(largest);
                    if (factor != 1.f) {
#pragma unroll
                        for (int b = 0; b < KB; ++b)
#pragma unroll
                            for (int d = 0; d < 2 * KD; ++d) acc_k[d][b] *= factor;
                    }
#pragma unroll
                    for (int b = 0; b < KB; ++b) {
                        dp[0][b] *= bs.scale;
                        dp[1][b] *= bs.scale;
                    }
                }
                Frag<T> p[KB][kOperands<T>], z[KB][kOperands<T>];
#pragma unroll
                for (int b = 0; b < KB; ++b) {
                    as_parts<T>(s[0][b], s[1][b], sc, p[b]);
                    as_parts<T>(dp[0][b], dp[1][b], sc, z[b]);
                }
                constexpr int kAtOnce = !kDeep ? 1 : KD <= 2 ? 2 * KD : KD; // operands
#pragma unroll
                for (int d0 = 0; d0 < 2 * KD; d0 += kAtOnce) {
                    Frag<T> f[kAtOnce], e[kAtOnce];
#pragma unroll
                    for (int d = 0; d < kAtOnce; ++d) {
                        f[d] = d0 + d < kEarly ? dc[d0 + d < kEarly ? d0 + d : kEarly] : TL::columns(dl, 32 * m, 16 * (d0 + d));
                        e[d] = TL::columns(ql, 32 * m, 16 * (d0 + d));
                    }
                    if constexpr (kDeep) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int d = 0; d < kAtOnce; ++d)
#pragma unroll
                        for (int part = 0; part < kOperands<T>; ++part)
#pragma unroll
                            for (int b = 0; b < KB; ++b) acc_v[d0 + d][b] = mma(f[d], p[b][part], acc_v[d0 + d][b]);
#pragma unroll
                    for (int d = 0; d < kAtOnce; ++d)
#pragma unroll
                        for (int part = 0; part < kOperands<T>; ++part)
#pragma unroll
                            for (int b = 0; b < KB; ++b) acc_k[d0 + d][b] = mma(e[d], z[b][part], acc_k[d0 + d][b]);
                }
            }
        if constexpr (kBuffers == 2) half ^= 1;
        else __syncthreads(); // (the tile has been read)
        if (n + 1 < end) stage(half, n + 1);
        ready(half);
    }
    const float of_k = kHalf ? a.scale * 0x1p-14f / bs.scale : a.scale, of_v = kHalf ? 0x1p-14f : 1.f;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
        if (key[b] >= a.s) continue;
        if (a.splits > 1) {
            const int64_t lines = (int64_t)a.n * a.batch * a.kv * a.s, line = ((int64_t)(at.particle * a.batch + at.batch) * a.kv + at.head) * a.s + key[b];
            float *const out = partial + (at.part * lines + line) * (64 * KD);
#pragma unroll
            for (int d = 0; d < 2 * KD; ++d) {
                *reinterpret_cast<f32x4 *>(out + 16 * d + 4 * g) = acc_k[d][b] * of_k;
                *reinterpret_cast<f32x4 *>(out + 32 * KD + 16 * d + 4 * g) = acc_v[d][b] * of_v;
            }
            continue;
        }
        T *const to_k = dk.at(at.particle, at.batch, at.head) + key[b] * dk.token, *const to_v = dv.at(at.particle, at.batch, at.head) + key[b] * dv.token;
#pragma unroll
        for (int d = 0; d < 2 * KD; ++d) {
            const int c = 16 * d + 4 * g;
            const float x[4] = {acc_k[d][b][0] * of_k, acc_k[d][b][1] * of_k, acc_k[d][b][2] * of_k, acc_k[d][b][3] * of_k};
            const float y[4] = {acc_v[d][b][0] * of_v, acc_v[d][b][1] * of_v, acc_v[d][b][2] * of_v, acc_v[d][b][3] * of_v};
            if (c < a.dim && dk.p) store_pack<T, 4>(to_k + c, a.dim - c, x);
            if (c < a.dim && dv.p) store_pack<T, 4>(to_v + c, a.dim - c, y);
        }
    }
}

// dq from the parts' sums, in order, and what eps puts on delta: a thread has four values of a line's ld (dq null, not wanted: delta alone,
// a thread a line).
template <class T> __global__ __launch_bounds__(256) void attention_query_sums_kernel(AttnArgs a, int ld, const float *partial, const float *row_sums, float *delta, Heads<T> dq)
{
    const int64_t lines = (int64_t)a.n * a.batch * a.heads * a.t;
    const int quads = dq.p ? ld / 4 : 1, each = kRestore<T> ? 2 * ld : ld;
    const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x, line = k / quads;
    const int c = (int)(k - line * quads) * 4;
    if (line >= lines || c >= a.dim) return;
    constexpr int U = kRestore<T> ? 4 : 8; // on their way together
    f32x4 sum = {0.f, 0.f, 0.f, 0.f}, mean = {0.f, 0.f, 0.f, 0.f};
    float eps = 0.f;
    for (int p0 = 0; p0 < a.splits; p0 += U) {
        f32x4 x[U], y[U];
        float z[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t p = min(p0 + u, a.splits - 1);
            const float *const from = partial + (p * lines + line) * each + c;
            if (dq.p) x[u] = *reinterpret_cast<const f32x4 *>(from);
            if constexpr (kRestore<T>) {
                if (dq.p) y[u] = *reinterpret_cast<const f32x4 *>(from + ld);
                z[u] = row_sums[p * lines + line];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p0 + u >= a.splits) continue;
            if (dq.p) sum += x[u];
            if constexpr (kRestore<T>) {
                if (dq.p) mean += y[u];
                eps += z[u];
            }
        }
    }
    if constexpr (kRestore<T>) {
        if (c == 0) delta[line] += eps;
        sum -= eps * mean;
    }
    if (!dq.p) return;
    const int i = (int)(line % a.t);
    const int64_t head = line / a.t;
    const int h = (int)(head % a.heads), b = (int)(head / a.heads % a.batch), particle = (int)(head / a.heads / a.batch);
    const float x[4] = {sum[0], sum[1], sum[2], sum[3]};
    store_pack<T, 4>(dq.at(particle, b, h) + i * dq.token + c, a.dim - c, x);
}

// dk and dv from the parts' sums, in order: a thread has four values of a line's two times ld.
template <class T> __global__ __launch_bounds__(256) void attention_key_sums_kernel(AttnArgs a, int ld, const float *partial, Heads<T> dk, Heads<T> dv)
{
    const int64_t lines = (int64_t)a.n * a.batch * a.kv * a.s;
    const int quads = ld / 2;
    const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x, line = k / quads;
    const int at = (int)(k - line * quads) * 4, which = at / ld, c = at - which * ld;
    if (line >= lines || c >= a.dim) return;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    constexpr int U = 8; // on their way together
    for (int p0 = 0; p0 < a.splits; p0 += U) {
        f32x4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = *reinterpret_cast<const f32x4 *>(partial + (min(p0 + u, a.splits - 1) * lines + line) * (2 * ld) + at);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p0 + u < a.splits) sum += x[u];
    }
    const Heads<T> &to = which ? dv : dk;
    if (!to.p) return;
    const int i = (int)(line % a.s);
    const int64_t head = line / a.s;
    const int h = (int)(head % a.kv), b = (int)(head / a.kv % a.batch), particle = (int)(head / a.kv / a.batch);
    const float x[4] = {sum[0], sum[1], sum[2], sum[3]};
    store_pack<T, 4>(to.at(particle, b, h) + i * to.token + c, a.dim - c, x);
}

// The rows' terms of the slopes' gradients from the parts': the sums of dz, and by turns those of dz and of P with the distances.
static __global__ __launch_bounds__(256) void attention_slope_rows_kernel(AttnArgs a, const float *row_sums, float *slope_rows)
{
    const int64_t lines = (int64_t)a.n * a.batch * a.heads * a.t, line = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (line >= lines) return;
    float z = 0.f, zf = 0.f, f = 0.f;
    for (int p = 0; p < a.splits; ++p) {
        z += row_sums[p * lines + line];
        zf += row_sums[(a.splits + 2 * p) * lines + line];
        f += row_sums[(a.splits + 2 * p + 1) * lines + line];
    }
    slope_rows[line] = z * f - zf;
}

// A slope's gradient: what its rows give, added up by one workgroup, in an order that is always the same.
static __global__ __launch_bounds__(256) void attention_slopes_kernel(AttnArgs a, const float *slope_rows, float *dslopes, int64_t stride, bool accumulate)
{
    __shared__ float sums[4];
    const int particle = blockIdx.x / a.heads, h = blockIdx.x - particle * a.heads;
    float sum = 0.f;
    for (int b = 0; b < a.batch; ++b) {
        const float *const rows = slope_rows + a.line(particle, b, h, 0);
        float part = 0.f;
        for (int i = threadIdx.x; i < a.t; i += 256) part += rows[i];
        sum += part;
    }
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        float *const to = dslopes + particle * stride + h;
        const float all = (sums[0] + sums[1]) + (sums[2] + sums[3]);
        *to = accumulate ? *to + all : all;
    }
}

} // namespace svgd
