// Which instances of the attention kernels a call takes and into how many parts its work goes: plain numbers, no HIP.  A: sizes and masks
// as AttnArgs has them.
#pragma once
#include <cstdint>

namespace svgd {

constexpr int kTileRows = 64; // streamed rows (or keys) in LDS at a time
constexpr int kAttnWaves = 4, kAttnBlock = 64 * kAttnWaves;
constexpr int64_t kMaxBlocks = ((int64_t)1 << 24) - 8; // (a launch has less than 2^32 threads)

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Blocks of 32 values of a head that the kernels are built for; heads of less than eight values have kernels of their own, numbered 0.
constexpr int dim_kind(int dim) { return dim < 8 ? 0 : (dim + 31) / 32; }

// Whether a wave can have two blocks of 16 rows (or keys) of its own, which halves what it reads from LDS, without running out of
// registers.  `size`: bytes of a value; `modified`: capped scores, or slopes.  (Capped scores of 16 bits could, but the waves that one
// block leaves room for are worth more: 4 x 2 x 2,000 x 8 heads over 2 of 64 fp16 forward 71 us with two, 62 with one; keys, 4 x 4 x 4,096
// x 8 heads of 64 bf16, causal, 1,071 and 1,012; measured with probabilities in one part.)
constexpr bool two_forward(int size, int kind, bool modified) { return !modified && (size == 2 || kind < 3); }
constexpr bool two_keys(int size, int kind, bool modified) { return !modified && kind < (size == 2 ? 3 : 2); }

// Workgroups with one block of 16 rows (or keys) for every wave.
template <class A> int64_t small_blocks(const A &a, int64_t size) { return (int64_t)a.n * a.batch * a.kv * ceil_div(size, 16 * kAttnWaves); }
// Two blocks to a wave where the workgroups are many all the same.  us with one and with two, heads of 64 bf16, 1,024 / 1,536 / 2,048 /
// 4,096 / 8,192 small workgroups:
//     forward, 200 keys            16.5, 16.1 / 22.7, 20.0 / 26.4, 25.8 / 45.0, 41.4 / 82.9, 74.9      2,048 keys            71, 65 / 102, 90 / 133, 119 / 255, 222 / 502, 431
//     forward, causal, 1,024 keys  29, 37 / 36, 48 / 46, 51 / 83, 82 / 159, 147                        causal, 2,048 keys    41, 49 / 77, 77 / 80, 79 / 145, 133 / 279, 250
//     keys, 200 of them            28.6, 23.3 / 33.7, 37.2 / 46.3, 41.6 / 82.7, 76.7 / 170, 161        2,048 of them         143, 102 / 179, 173 / 236, 202 / 463, 394 / 938, 796
//     keys, causal, 200            24.9, 21.9 / 29.6, 35.2 / 37.7, 41.0 / 65.8, 71.9 / 130, 144        causal, 2,048         70, 80 / 119, 115 / 126, 119 / 250, 224 / 500, 466
// (heads of 32 and 96 gain up to 17 % less from two, of 128 up to 15 % more).  With queries of their own, which two blocks cost more
// registers, always one (with one or two and four products, 4 x 2 x 4,096 x 16 heads of 64 causal: 671 / 684).
constexpr int64_t kManyKeys = 4096;
template <class A> bool many_forward(const A &a)
{
    const bool even = !a.causal && !a.documents;
    return small_blocks(a, a.rows) >= (even ? 1024 : a.s >= 2048 ? 1536 : 4096);
}
template <class A> bool many_keys(const A &a) { return small_blocks(a, a.s) >= kManyKeys; }

// Where workgroups with rows (or keys) of their own are few, the streamed ones go in parts, whose sums are added up afterwards.  In units
// of a tile's time a workgroup takes its tiles and one for the time until the first is there, and all of them take rounds of kAtATime.
// Masks leave some of the workgroups less, how much on an average is `share`; the card then works on until the longest is done, and as fast
// as kAtOnce workgroups that wait for nothing.  Parts' sums cost a launch. (us of the keys' kernel with the sums in 1 / 2 / 3 / 4 parts: 4
// x 2 x 2,000 x 8 heads over 2 of 64 fp16, causal, capped, 7 documents, the longest of 939 tokens, 192 / 118 / 109 / 118, of like lengths
// 89 / 92 / 87 / 99; 4 x 2 x 1,000 x 8 over 4 of 64 bf16 causal 63 / 51 / 55 / 59; 3 x 1,500 x 8 over 4 of 64 fp32 causal 222 / 126 / 98 /
// 99; 8 x 2 x 512 x 4 of 64 bf16 causal 23 / 32 / 35 / 41; 1 x 4,000 x 4 of 128 bf16 154 / 118 / 133 / 125.  The rule takes 2, 2, 3, 1 and
// 2.)
constexpr int64_t kAtATime = 512;
constexpr double kAtOnce = 341;
template <class A> int parts_for(const A &a, int64_t own, int64_t streamed)
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
// Few rows.  us with 512 / 1,024 / 2,048 / 4,096 workgroups wanted, the join included: 8 x 4 x 1 over 8,192 x 4 heads of 128 bf16, 16 query
// heads, 92.8 / 91.9 / 93.8 / 104.8; 8 x 8 x 1 over 4,096 x 4 of 128 91.7 / 89.1 / 86.9 / 90.9; 32 x 8 x 1 over 2,048 x 4 of 64 fp16 89 /
// 87 / 87 / 84; one sequence over 8,192 x 8 of 128 16 whatever is wanted.
constexpr int64_t kFewBlocks = 1024;
template <class A> bool few_rows(const A &a) { return a.rows <= 16; }
template <class A> int forward_splits(const A &a)
{
    if (!few_rows(a)) return parts_for(a, a.rows, a.s);
    // two tiles of 32 keys for every wave at least
    const int64_t blocks = small_blocks(a, a.rows), most = a.s / (2 * kAttnWaves * 32), wanted = ceil_div(kFewBlocks, blocks < 1 ? 1 : blocks);
    const int64_t parts = wanted < most ? wanted : most;
    return (int)(parts < 1 ? 1 : parts > 64 ? 64 : parts);
}
template <class A> int query_splits(const A &a) { return parts_for(a, a.rows, a.s); }
template <class A> int key_splits(const A &a) { return parts_for(a, a.s, a.rows); }

} // namespace svgd
