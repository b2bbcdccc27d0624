// Which tiles a linear map takes, and into how many parts its columns go: plain numbers, no HIP.  Kinds, costs and limits are those of
// ffn_rules.hpp.
#pragma once
#include "ffn_rules.hpp"

namespace svgd {

// What a launch takes (ffn_rules.hpp says in what): of the kinds and of one, two or four parts at 14 shapes (1 to 32 particles of 40 to
// 16,000 rows, 64 to 2,000 wide), fp32 and bf16, forward finds the fastest or one within 8 % of it, backward one within 14 %.  (With the
// rates of the feed-forward block's products 5 x 1,003 x 333 x 501 fp32 forward took 39 us, so 29; 8 x 1,576 x 384 x 1,152 fp32 backward
// 202 and 172.)
constexpr Rates kOfLinear = {{1.0, 0.61, 0.42}, 1.0, 8.8, 0.1, 3.7e6};
constexpr Rates kOfLinearGradients = {{1.0, 0.73, 0.54}, 0.78, 6.2, 4.0, 12e6};

inline int64_t linear_ld(int64_t out) { return (out + 3) / 4 * 4; } // rows of z, of dz and of parts' sums start on 16 bytes

struct LinearForwardPlan {
    bool thin;
    Choice tile;
    LinearForwardPlan(int n, int64_t rows, int64_t width, int64_t out)
        : thin(rows <= kThinRows), tile(choose(kOfLinear, n, out, rows, width, 1, n * rows * out))
    {
        if (thin) tile.parts = 1;
    }
    bool fits() const { return thin || tile.parts; }
    size_t scratch(int n, int64_t rows, int64_t out) const { return tile.parts > 1 ? (size_t)tile.parts * n * rows * linear_ld(out) * 4 : 0; }
};

// dx and the weight's gradient: tiles of one kind, in one launch.  The bias's gradient: `sums` parts of the rows.  Without an activation dz
// is dy and has no place in scratch memory.
struct LinearBackwardPlan {
    TileKind kind = kLarge;
    int input_parts = 1, param_parts = 0, sums;
    int64_t sum_rows; // rows of each
    size_t dz_floats, input_floats, param_floats, sum_floats;
    LinearBackwardPlan(int n, int64_t rows, int64_t width, int64_t out, bool activation = true)
    {
        double least = 1e30;
        for (int kd = 0; kd < kTileKinds; ++kd) {
            const KindOf &k = kKinds[kd];
            const int64_t params = n * tiles(width, k.i) * tiles(out, k.j), input = n * tiles(width, k.i) * tiles(rows, k.j);
            if (!launchable((TileKind)kd, blocks_for(params) + blocks_for(input))) continue;
            for (int pp = 1; pp <= 32 && (pp == 1 || (rows / pp >= 4 * kTileK && params * pp <= 1024)); pp *= 2)
                for (int ip = 1; ip <= 32 && (ip == 1 || (out / ip >= 4 * kTileK && input * ip <= 1024)); ip *= 2) {
                    const double of_params = steps_of(kOfLinearGradients, rows, pp), of_input = steps_of(kOfLinearGradients, out, ip);
                    const double c = launch_cost(kOfLinearGradients, (TileKind)kd, params * pp + input * ip, (double)(params * pp) * of_params + (double)(input * ip) * of_input,
                                                 of_params > of_input ? of_params : of_input) +
                                     reduce_cost(kOfLinearGradients, pp, n * width * out) + reduce_cost(kOfLinearGradients, ip, n * rows * width);
                    if (c < least) {
                        least = c;
                        kind = (TileKind)kd;
                        param_parts = pp;
                        input_parts = ip;
                    }
                }
        }
        const int64_t groups = n * tiles(out, 256), wanted = tiles(1024, (int)(groups < 1024 ? groups : 1024));
        int64_t s = rows / 16 < wanted ? rows / 16 : wanted;
        s = s < 1 ? 1 : s > 128 ? 128 : s;
        sum_rows = rows > 0 ? (rows + s - 1) / s : 1;
        sums = rows > 0 ? (int)((rows + sum_rows - 1) / sum_rows) : 0;
        dz_floats = activation ? (size_t)n * rows * linear_ld(out) : 0;
        input_floats = input_parts > 1 ? (size_t)input_parts * n * rows * linear_ld(width) : 0;
        param_floats = param_parts > 1 ? (size_t)param_parts * n * width * out : 0;
        sum_floats = sums > 1 ? (size_t)sums * n * out : 0;
    }
    bool fits() const { return param_parts > 0; }
    size_t scratch() const { return (dz_floats + input_floats + param_floats + sum_floats + 16) * 4; } // (each begins on 16 bytes)
};

} // namespace svgd
