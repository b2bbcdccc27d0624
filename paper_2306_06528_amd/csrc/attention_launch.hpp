// What a call of attention launches, by sizes alone.  The kernels' instances are compiled type by type (attention_*_<type>.hip).
#pragma once
#include "attention_common.hpp"

namespace svgd {

struct AttnCall {
    AttnArgs a;
    svgd_heads q, k, v, o, d_o, dq, dk, dv;
    const float *lse, *delta;
    float *lse_out, *partial, *partial_lse, *slope_rows;
    hipStream_t stream;
};

template <class T> Heads<const T> in(const svgd_heads &h) { return {(const T *)h.data, h.particle_stride, h.batch_stride, h.token_stride, h.head_stride}; }
template <class T> Heads<T> out(const svgd_heads &h) { return {(T *)h.data, h.particle_stride, h.batch_stride, h.token_stride, h.head_stride}; }

constexpr int64_t kMaxBlocks = ((int64_t)1 << 24) - 8; // (a launch has less than 2^32 threads)

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups with one block of 16 rows (or keys) for every wave.
inline int64_t small_blocks(const AttnArgs &a, int64_t size) { return (int64_t)a.n * a.batch * a.kv * ceil_div(size, 16 * kAttnWaves); }
// Two blocks to a wave where the workgroups are many all the same.  us with one and with two, 8 x 8 x 197 x 6 heads of 64 bf16 (1,536 small workgroups) and 4 x 2 x 4,096 x 16 heads of 64 causal (8,192): forward
// 21 / 18 and 457 / 392, keys 34.7 / 40 and 999 / 915; with queries of their own, which two blocks cost more registers, 27.9 / 30.3 and 671 / 684, so always one.
constexpr int64_t kManyForward = 1024, kManyKeys = 4096;

// Where workgroups with rows (or keys) of their own are few, the streamed ones go in parts, whose sums are added up afterwards: as many as make the shortest way of a workgroup's tiles, the time until its first one
// is there (one tile's) and, with parts, the sums' own launch, times the rounds of kAtATime workgroups.  (3 x 2 x 333 x 6 heads of 40 fp32, 192 workgroups of 6 tiles: 3 parts, which make two rounds, 20 us, 2 parts 15.)
constexpr int64_t kAtATime = 512;
inline int parts_for(const AttnArgs &a, int64_t own, int64_t streamed)
{
    const int64_t blocks = small_blocks(a, own), tiles = ceil_div(streamed, kTileRows);
    if (blocks == 0 || blocks >= kAtATime) return 1;
    int64_t best = 1, least = tiles + 1;
    for (int64_t parts = 2; parts <= 64 && 2 * parts <= tiles; ++parts) {
        const int64_t cost = ceil_div(blocks * parts, kAtATime) * (ceil_div(tiles, parts) + 1) + 1;
        if (cost < least) {
            least = cost;
            best = parts;
        }
    }
    return (int)best;
}
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
