// Which tiles a call of the gated feed-forward block takes, and into how many parts its columns go: plain numbers, no HIP.
#pragma once
#include <cstddef>
#include <cstdint>

namespace svgd {

constexpr int kTileK = 32; // columns of both operands per step

inline int64_t hidden_ld(int64_t hidden) { return (hidden + 31) / 32 * 32; } // rows of the buffers start on 128 bytes

inline int64_t tiles(int64_t size, int tile) { return (size + tile - 1) / tile; }

// ---------------------------------------------------------------------------------------------
// Which tiles, and into how many parts the columns go: by sizes alone, the same for every type.  (The smallest tiles of g, u and dh take 164 registers for
// bf16 activations, 192 for fp32, so half as many more workgroups run at a time: the rule reckons with fp32.)
// ---------------------------------------------------------------------------------------------
enum TileKind { kLarge, kSmall, kTiny, kTileKinds };
struct KindOf {
    int i, j, threads, at_a_time; // threads of a workgroup, workgroups that run at a time on the whole part
};
constexpr KindOf kKinds[kTileKinds] = {{256, 128, 256, 512}, {128, 64, 128, 1024}, {64, 32, 64, 2048}};

// Tiles of one grid are launched by eights, one for each die.  A launch has less than 2^32 threads.
constexpr int kDies = 8;
inline int64_t blocks_for(int64_t tile_count) { return (tile_count + kDies - 1) / kDies * kDies; }
inline bool launchable(TileKind kind, int64_t blocks) { return blocks * kKinds[kind].threads < (int64_t)1 << 32; }

// What a launch takes, in steps (32 columns) of a large tile on a full CU (4.4 us fp32, 3 us bf16): workgroups of `longest` steps and `work` steps
// in all.  Fewer than run at a time take as long as the longest, and that is `half` times as long where a CU has only half of them;
// of more, the last ones end 0.4 of their length late.
struct Rates {
    double step[kTileKinds], half, start; // a tile's step; see above; steps until a workgroup's first rows are there, and for its results
    double launch, bytes;                 // what adding up parts' sums costs: a launch, and the bytes that it moves in a step's time
};
// g and u, dh: at 15 shapes (1 to 40 particles of 64 to 16,000 rows, 64 to 1,024 wide) this finds the fastest or one within 5 % of it.
constexpr Rates kUsual = {{1.0, 0.6, 0.35}, 0.6, 4.0, 0.0, 1.0}; // (never in parts)
// y = h down^T: the one product whose operands both lie along the columns, both of three parts.  Small tiles cost more there (of 15 shapes, 1 to 40 particles
// of 64 to 16,000 rows, 64 to 1,024 wide, this finds the fastest or one within 5 % of it at 14 and takes 7 % more at one; with the usual ones forward would take 8 x 1,576 x 384 x
// 1,024 bf16 166 us for 155, 2 x 3,000 x 768 x 2,048 fp32 351 for 297).
constexpr Rates kOfDown = {{1.0, 0.6, 0.5}, 0.8, 3.0, 0.6, 16e6};
// The gradients, tiles of dx and of the parameters in one launch: workgroups of other lengths side by side, results of four bytes each.  Of all kinds
// and parts at 27 shapes (1 to 64 particles of 50 to 16,000 rows, 48 to 1,024 wide) this finds the fastest or one within 5 % of it at 23 and
// never takes more than 17 % more.
constexpr Rates kOfGradients = {{1.0, 0.62, 0.4}, 0.9, 10.0, 0.3, 6e6};
inline double launch_cost(const Rates &r, TileKind kind, int64_t workgroups, double work, double longest)
{
    const int at_a_time = kKinds[kind].at_a_time;
    if (workgroups <= at_a_time) return longest * r.step[kind] * (2 * workgroups <= at_a_time ? r.half : 1.0);
    return (work / at_a_time + 0.4 * longest) * r.step[kind];
}
inline double steps_of(const Rates &r, int64_t columns, int parts) { return (double)(((columns + parts - 1) / parts + kTileK - 1) / kTileK) + r.start; }
// Parts' sums are written and read once more.
inline double reduce_cost(const Rates &r, int parts, int64_t floats) { return parts > 1 ? r.launch + (double)floats * parts * 8.0 / r.bytes : 0.0; }

struct Choice {
    TileKind kind;
    int parts; // 0: there are more tiles than a launch takes, of every kind
};

// The cheapest kind for C[j][i] of each of n particles over `columns` columns, and with `sums` (floats in a part's sums, 0: not
// to be split) the cheapest number of parts.
inline Choice choose(const Rates &r, int n, int64_t i, int64_t j, int64_t columns, int per_i, int64_t sums)
{
    Choice best{kLarge, 0};
    double least = 1e30;
    for (int kind = 0; kind < kTileKinds; ++kind) {
        const int64_t t = n * tiles(i, kKinds[kind].i / per_i) * tiles(j, kKinds[kind].j);
        if (!launchable((TileKind)kind, blocks_for(t))) continue;
        for (int parts = 1; parts <= (sums ? 32 : 1) && (parts == 1 || (columns / parts >= 4 * kTileK && t * parts <= 1024)); parts *= 2) {
            const double steps = steps_of(r, columns, parts), c = launch_cost(r, (TileKind)kind, t * parts, (double)(t * parts) * steps, steps) + reduce_cost(r, parts, sums);
            if (c < least) {
                least = c;
                best = {(TileKind)kind, parts};
            }
        }
    }
    return best;
}

// Up to so many rows per particle every weight is read once, by a wave of its own (ffn_thin_kernels.hpp).  Forward: 8 x 17 rows, 384 x 1,024 fp32, 14 us, in
// tiles 26, 8 x 32 rows 16 and 28; the worst, 8 x 32 rows, 1,024 x 2,730 bf16, 63 and 61.  dg and du: these and the gradients of the parameters, 4 x 16 rows, 384 x 1,024 fp32, 19 and
// 29, 1 x 32 rows, 3,000 x 8,000, 159 and 218, 64 x 32 rows, 128 x 341, 32 and 31.
// Forward up to 64 rows where the tiles of g and u are few: 1 x 64 rows, 1,024 x 2,730 fp32, 22 tiles, 30 and 51, 8 x 64 rows, 384 x 1,024, 64 tiles, 23 and 29,
// 4 x 64 rows, 1,024 x 2,730, 88 tiles, 55 and 68, but 16 x 64 rows, 512 x 1,400, 176 tiles, 61 both, 40 x 64 rows, 256 x 700, 240 tiles, 52 and 41.
constexpr int64_t kThinRows = 32;
inline bool thin_forward_rows(int n, int64_t rows, int64_t hidden)
{
    return rows <= kThinRows || (rows <= 64 && n * tiles(hidden, kKinds[kLarge].i / 2) < 128);
}

// The same for dx, whose waves have all of the hidden width to go through.  With gradients of parameters, in whose launch dx's tiles find room, only in narrow
// layers: both, 3 x 16 rows, 64 x 200 fp32, 15 us, as tiles 18, 64 x 16 rows, 96 x 250, 26 and 31, but 64 x 16 rows, 128 x 341, 36 both, 8 x 16 rows, 384 x 1,024, 36 and 35, with 32 rows 42 and 35,
// 1 x 32 rows, 1,024 x 2,730, 72 and 48.  dx alone, unless few waves would have long ways: 8 x 16 rows, 384 x 1,024, 17 and 21, 40 x 16 rows, 256 x 700, 34 and 50, but
// 2 x 16 rows, 200 x 1,500, 31 and 20, 1 x 16 rows, 256 x 16,000, 120 and 47.
inline bool thin_input_rows(int n, int64_t rows, int64_t width, int64_t hidden, bool params_too)
{
    if (rows == 0 || rows > kThinRows) return rows == 0;
    if (params_too) return width * hidden <= 1 << 15;
    return hidden <= 1024 || hidden <= 64 * n * tiles(width, 32);
}

inline int64_t width_ld(int64_t width) { return (width + 3) / 4 * 4; }

struct ForwardPlan {
    bool thin;
    Choice gate_up, down;
    ForwardPlan(int n, int64_t rows, int64_t width, int64_t hidden)
        : thin(thin_forward_rows(n, rows, hidden)), gate_up(choose(kUsual, n, hidden, rows, width, 2, 0)),
          down(choose(kOfDown, n, width, rows, hidden, 1, n * rows * width))
    {
        if (thin) down.parts = 1;
    }
    bool fits() const { return thin || (gate_up.parts && down.parts); } // otherwise nothing is launched
    size_t scratch(int n, int64_t rows, int64_t width) const { return down.parts > 1 ? (size_t)down.parts * n * rows * width_ld(width) * 4 : 0; }
};

// The gradients' tiles are of one kind, being of one launch.  input_parts is 1 or even, see input_grad_tile.  params_too: gradients of parameters are wanted.
struct BackwardPlan {
    Choice hidden;
    TileKind gradients = kLarge;
    int input_parts = 1, param_parts = 0;
    bool thin, thin_input; // dg and du, dx by a wave for every weight
    size_t hidden_floats, input_floats, gate_floats, down_floats;
    BackwardPlan(int n, int64_t rows, int64_t width, int64_t hid, bool params_too)
        : hidden(choose(kUsual, n, hid, rows, width, 1, 0)), thin(rows <= kThinRows), thin_input(thin_input_rows(n, rows, width, hid, params_too))
    {
        double least = 1e30;
        for (int kind = 0; kind < kTileKinds; ++kind) {
            const KindOf &k = kKinds[kind];
            const int64_t params = 3 * n * tiles(width, k.i) * tiles(hid, k.j), input = !thin_input ? n * tiles(width, k.i) * tiles(rows, k.j) : 0;
            if (thin && kind == kLarge) continue; // (one step each: 8 x 8 rows, 384 x 1,024 fp32, all gradients 44 us, small ones 35, 40 x 8 rows, 256 x 700, 89 and 70; never the best by more than 2 %)
            if (!launchable((TileKind)kind, blocks_for(params / 3 * 2) + blocks_for(params / 3) + blocks_for(input))) continue;
            for (int pp = 1; pp <= 32 && (pp == 1 || (rows / pp >= 4 * kTileK && params * pp <= 1024)); pp *= 2)
                for (int ip = 1; ip <= 32 && (ip == 1 || (2 * hid / ip >= 4 * kTileK && input * ip <= 1024 && input > 0)); ip *= 2) {
                    const double of_params = steps_of(kOfGradients, rows, pp), of_input = input ? steps_of(kOfGradients, 2 * hid, ip) : 0.0;
                    const double c = launch_cost(kOfGradients, (TileKind)kind, params * pp + input * ip,
                                                 (double)(params * pp) * of_params + (double)(input * ip) * of_input, of_params > of_input ? of_params : of_input) +
                                     reduce_cost(kOfGradients, pp, 3 * n * width * hid) + (pp > 1 ? kOfGradients.launch : 0.0) +
                                     reduce_cost(kOfGradients, ip, n * rows * width);
                    if (c < least) {
                        least = c;
                        gradients = (TileKind)kind;
                        param_parts = pp;
                        input_parts = ip;
                    }
                }
        }
        hidden_floats = (size_t)n * rows * hidden_ld(hid);
        input_floats = input_parts > 1 ? (size_t)input_parts * n * rows * width_ld(width) : 0;
        gate_floats = param_parts > 1 ? (size_t)param_parts * n * 2 * width * hid : 0;
        down_floats = param_parts > 1 ? (size_t)param_parts * n * width * hid : 0;
    }
    bool fits() const { return (thin || hidden.parts) && param_parts; }
    size_t scratch() const { return (2 * hidden_floats + input_floats + gate_floats + down_floats + 16) * 4; } // (each begins on 16 bytes)
};
inline size_t aligned4(size_t floats) { return (floats + 3) & ~(size_t)3; }

} // namespace svgd
