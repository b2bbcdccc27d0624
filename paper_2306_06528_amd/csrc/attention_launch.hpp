// What a call of attention launches, by sizes alone.  The kernels' instances are compiled type by type (attention_*_<type>.hip).
#pragma once
#include "attention_common.hpp"

namespace svgd {

struct AttnCall {
    AttnArgs a;
    svgd_heads q, k, v, o, d_o, dq, dk, dv;
    const float *lse, *delta;
    float *lse_out, *partial, *partial_lse, *slope_rows, *row_sums;
    hipStream_t stream;
};

template <class T> Heads<const T> in(const svgd_heads &h) { return {(const T *)h.data, h.particle_stride, h.batch_stride, h.token_stride, h.head_stride}; }
template <class T> Heads<T> out(const svgd_heads &h) { return {(T *)h.data, h.particle_stride, h.batch_stride, h.token_stride, h.head_stride}; }

constexpr int64_t kMaxBlocks = ((int64_t)1 << 24) - 8; // (a launch has less than 2^32 threads)

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups with one block of 16 rows (or keys) for every wave.
inline int64_t small_blocks(const AttnArgs &a, int64_t size) { return (int64_t)a.n * a.batch * a.kv * ceil_div(size, 16 * kAttnWaves); }
// Two blocks to a wave where the workgroups are many all the same.  us with one and with two, 8 x 8 x 197 x 6 heads of 64 bf16 (1,536 small workgroups) and 4 x 2 x 4,096 x 16 heads of 64 causal (8,192): forward
// 21 / 18 and 457 / 392, keys 34.7 / 40 and 999 / 915; with queries of their own, which two blocks cost more registers, 27.9 / 30.3 and 671 / 684, so always one.  Masked calls, whose workgroups differ, are better off with
// twice as many while these are few or short (64 bf16, causal: 1,024 of 2,048 keys 38 / 45, 1,536 of 1,024 keys 34 / 43 and of 4,096 99 / 91, 2,048 of 1,024 keys 42 / 45 and of 4,096 107 / 93, 4,096 of 1,024 keys 69 / 69).
constexpr int64_t kManyKeys = 4096;
inline bool many_forward(const AttnArgs &a)
{
    const bool even = !a.causal && !a.documents;
    return small_blocks(a, a.rows) >= (even ? 1024 : a.s >= 2048 ? 1536 : 4096);
}

// Where workgroups with rows (or keys) of their own are few, the streamed ones go in parts, whose sums are added up afterwards.  In units of a tile's time a workgroup takes its tiles and one for the time until the
// first is there, and all of them take rounds of kAtATime.  Masks leave some of the workgroups less, how much on an average is `share`; the card then works on until the longest is done, and as fast as kAtOnce
// workgroups that wait for nothing.  Parts' sums cost a launch.  (us of the keys' kernel in 1 / 2 / 3 / 4 parts, and of the sums: 4 x 2 x 2,000 x 8 heads over 2 of 64 fp16, causal, capped, 7 documents 226 / 129 / 113 / 122 and
// 11; 4 x 2 x 1,000 x 8 over 4 of 64 bf16 causal 63 / 42 / 45 / 48 and 11; 3 x 1,500 x 8 over 4 of 64 fp32 causal 235 / 133 / 104 / 106 and 8; 8 x 2 x 512 x 4 of 64 bf16 causal 22.6 / 21.8 / 23 / 28 and 11.)
constexpr int64_t kAtATime = 512;
constexpr double kAtOnce = 341;
inline int parts_for(const AttnArgs &a, int64_t own, int64_t streamed)
{
    const int64_t blocks = small_blocks(a, own), tiles = ceil_div(streamed, kTileRows);
    const bool even = !a.causal && !a.documents;
    if (blocks == 0 || blocks >= (even ? 1 : 2) * kAtATime) return 1;
    const double share = a.documents ? 0.5 : 1 - 0.5 * (a.t < a.s ? a.t : a.s) / a.s;
    int64_t best = 1;
    double least = 1e30;
    for (int64_t parts = 1; parts == 1 || (parts <= 64 && 2 * parts <= tiles); ++parts) {
        const double longest = (double)(ceil_div(tiles, parts) + 1);
        double cost = ceil_div(blocks * parts, kAtATime) * longest + (parts > 1 ? 1 : 0);
        if (!even) {
            const double all = (double)(blocks * parts) * (share * tiles / parts + 1) / kAtOnce;
            cost = (all > longest ? all : longest) + (parts > 1 ? 2 : 0);
        }
        if (cost < least) {
            least = cost;
            best = parts;
        }
    }
    return (int)best;
}
// (8 x 4 x 1 over up to 8,192 x 4 heads of 128 bf16, 16 query heads: 512 workgroups 81.2 us, 1,024 79.2, and the join 4.6 either way)
constexpr int64_t kFewBlocks = 1024;
inline bool few_rows(const AttnArgs &a) { return a.rows <= 16; }
inline int forward_splits(const AttnArgs &a)
{
    if (!few_rows(a)) return parts_for(a, a.rows, a.s);
    // two tiles of 32 keys for every wave at least
    const int64_t blocks = small_blocks(a, a.rows), most = a.s / (2 * kAttnWaves * 32), wanted = ceil_div(kFewBlocks, blocks);
    const int64_t parts = wanted < most ? wanted : most;
    return (int)(parts < 1 ? 1 : parts > 64 ? 64 : parts);
}
inline int query_splits(const AttnArgs &a) { return parts_for(a, a.rows, a.s); }
inline int key_splits(const AttnArgs &a) { return parts_for(a, a.s, a.rows); }

// Tiles of `own` rows each of `size`, the streamed ones in `splits` parts; the workgroups' numbers.
inline void set_grid(AttnArgs &a, int64_t size, int own, int splits)
{
    a.tiles = (int)ceil_div(size, own);
    a.splits = splits;
    a.total = (int)((int64_t)a.n * a.batch * a.kv * a.tiles * splits);
    a.per_die = (a.total + 7) / 8;
}

inline int padded_dim(const AttnArgs &a) { return (a.dim + 31) / 32 * 32; }

template <class T, class F> int with_dim(int dim, F f)
{
    using std::integral_constant;
    if (dim < 8) return f(integral_constant<int, 0>{});
    if (dim <= 32) return f(integral_constant<int, 1>{});
    if (dim <= 64) return f(integral_constant<int, 2>{});
    if (dim <= 96) return f(integral_constant<int, 3>{});
    return f(integral_constant<int, 4>{});
}
template <class F> int with_truth(bool b, F f) { return b ? f(std::true_type{}) : f(std::false_type{}); }

inline bool modified_scores(const AttnArgs &a) { return a.cap > 0.f || a.slopes; }
inline int launched_ok() { return hipGetLastError() == hipSuccess ? SVGD_OK : SVGD_ERR_DEVICE; }

template <class T> int attention_forward(AttnCall &c);
template <class T> int attention_queries(AttnCall &c);
template <class T> int attention_keys(AttnCall &c);

} // namespace svgd
