// Which tiles a call takes, into how many parts its columns go, and the launches of both passes.  The kernels' instances are compiled
// type by type (layers_ffn_*.hip).
#pragma once
#include "ffn_thin_kernels.hpp"

namespace svgd {

inline int64_t hidden_ld(int64_t hidden) { return (hidden + 31) / 32 * 32; } // rows of the buffers start on 128 bytes

inline int64_t tiles(int64_t size, int tile) { return (size + tile - 1) / tile; }

// ---------------------------------------------------------------------------------------------
// Which tiles, and into how many parts the columns go: by sizes alone, the same for every type
// ---------------------------------------------------------------------------------------------
enum TileKind { kLarge, kSmall, kTiny, kTileKinds };
typedef Tile<4, 8> LargeTile;
typedef Tile<2, 4> SmallTile;
typedef Tile<1, 2> TinyTile;
struct KindOf {
    int i, j, at_a_time; // workgroups that run at a time on the whole part
};
constexpr KindOf kKinds[kTileKinds] = {{LargeTile::kI, LargeTile::kJ, 512}, {SmallTile::kI, SmallTile::kJ, 1024}, {TinyTile::kI, TinyTile::kJ, 2048}};

// What a launch takes, in steps (32 columns) of a large tile on a full CU (4.4 us fp32, 3 us bf16): workgroups of `longest` steps and `work` steps
// in all.  Fewer than run at a time take as long as the longest, and that is `half` times as long where a CU has only half of them;
// of more, the last ones end 0.4 of their length late.
struct Rates {
    double step[kTileKinds], half, start; // a tile's step; see above; steps until a workgroup's first rows are there, and for its results
    double launch, bytes;                 // what adding up parts' sums costs: a launch, and the bytes that it moves in a step's time
};
// g and u, dh: at 15 shapes (1 to 40 particles of 64 to 16,000 rows, 64 to 1,024 wide) this finds the fastest or one within 5 % of it.
constexpr Rates kUsual = {{1.0, 0.6, 0.35}, 0.6, 4.0, 0.0, 1.0}; // (never in parts)
// y = h down^T: the one product whose operands both lie along the columns, h of three parts.  Small tiles cost more there (at 15 shapes, 1 to 40 particles
// of 64 to 16,000 rows, 64 to 1,024 wide, this finds the fastest or one within 5 % of it; with the usual ones forward took 8 x 1,576 x 384 x
// 1,024 bf16 146 us for 134, 2 x 3,000 x 768 x 2,048 fp32 345 for 299).
constexpr Rates kOfDown = {{1.0, 0.6, 0.5}, 0.8, 3.0, 0.6, 16e6};
// The gradients, tiles of dx and of the parameters in one launch: workgroups of other lengths side by side, results of four bytes each.  Of all kinds
// and parts at 27 shapes (1 to 64 particles of 50 to 16,000 rows, 48 to 1,024 wide) this finds the fastest or one within 5 % of it at 23 and
// never takes more than 20 % more; with the usual rates and kOfDown's reductions these would be 17 and 22 %.
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
    int parts;
};

// The cheapest kind for C[j][i] of each of n particles over `columns` columns, and with `sums` (floats in a part's sums, 0: not
// to be split) the cheapest number of parts.
inline Choice choose(const Rates &r, int n, int64_t i, int64_t j, int64_t columns, int per_i, int64_t sums)
{
    Choice best{kLarge, 1};
    double least = 1e30;
    for (int kind = 0; kind < kTileKinds; ++kind) {
        const int64_t t = n * tiles(i, kKinds[kind].i / per_i) * tiles(j, kKinds[kind].j);
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

template <class F> int with_tile(TileKind kind, F f)
{
    return kind == kLarge ? f(LargeTile{}) : kind == kSmall ? f(SmallTile{}) : f(TinyTile{});
}

// Up to so many rows per particle every weight is read once, by a wave of its own (ffn_thin_kernels.hpp): 8 x 17 rows, 384 x 1,024 fp32, forward 15 us,
// in tiles 27, 8 x 32 rows 16 and 28; backward of 8 x 17 rows 41, in tiles (of the time) 179.  Forward up to 64 rows where the tiles of g and u are few: 1 x 64
// rows, 1,024 x 2,730 fp32, 22 tiles, 29 and 51, 8 x 64 rows, 384 x 1,024, 64 tiles, 23 and 29, but 16 x 64 rows, 512 x 1,400 bf16, 176 tiles, 50 and 45,
// 40 x 64 rows, 256 x 700, 240 tiles, 49 and 36.
constexpr int64_t kThinRows = 32;
inline bool thin_forward_rows(int n, int64_t rows, int64_t hidden)
{
    return rows <= kThinRows || (rows <= 64 && n * tiles(hidden, LargeTile::kI / 2) < 128);
}

inline int64_t width_ld(int64_t width) { return (width + 3) / 4 * 4; }

struct ForwardPlan {
    Choice gate_up, down;
    ForwardPlan(int n, int64_t rows, int64_t width, int64_t hidden)
        : gate_up(choose(kUsual, n, hidden, rows, width, 2, 0)), down(choose(kOfDown, n, width, rows, hidden, 1, n * rows * width))
    {
        if (thin_forward_rows(n, rows, hidden)) down.parts = 1;
    }
    size_t scratch(int n, int64_t rows, int64_t width) const { return down.parts > 1 ? (size_t)down.parts * n * rows * width_ld(width) * 4 : 0; }
};

// The gradients' tiles are of one kind, being of one launch.  input_parts is 1 or even, see input_grad_tile.
struct BackwardPlan {
    Choice hidden;
    TileKind gradients = kLarge;
    int input_parts = 1, param_parts = 1;
    size_t hidden_floats, input_floats, gate_floats, down_floats;
    BackwardPlan(int n, int64_t rows, int64_t width, int64_t hid) : hidden(choose(kUsual, n, hid, rows, width, 1, 0))
    {
        double least = 1e30;
        for (int kind = 0; kind < kTileKinds; ++kind) {
            const KindOf &k = kKinds[kind];
            const int64_t params = 3 * n * tiles(width, k.i) * tiles(hid, k.j), input = rows > kThinRows ? n * tiles(width, k.i) * tiles(rows, k.j) : 0;
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
    size_t scratch() const { return (2 * hidden_floats + input_floats + gate_floats + down_floats + 16) * 4; } // (each begins on 16 bytes)
};
inline size_t aligned4(size_t floats) { return (floats + 3) & ~(size_t)3; }

struct FfnCall {
    int dtype, activation, n;
    FfnShape s;
    Params gate, up, down;
    hipStream_t stream;
};

template <class T> Rows<const T> in(const svgd_rows &r) { return {(const T *)r.data, r.particle_stride, r.row_stride}; }
template <class T> Rows<T> out(const svgd_rows &r) { return {(T *)r.data, r.particle_stride, r.row_stride}; }
inline int launched() { return hipGetLastError() == hipSuccess ? SVGD_OK : SVGD_ERR_DEVICE; }

template <class T> int reduce_rows(const FfnCall &c, const float *partial, int parts, const Rows<T> &y)
{
    const int64_t quads = c.n * c.s.rows * c.s.width_ld / 4;
    reduce_rows_kernel<T><<<(unsigned)tiles(quads, 256), 256, 0, c.stream>>>(c.s, partial, parts, y);
    return launched();
}

template <class T, int ACT, int JB> int thin_forward(const FfnCall &c, const svgd_rows &x, const svgd_rows &y, float *h, float *g, float *u, bool save)
{
    const ThinGrid first(c.s.hidden, 16), second(c.s.width, 16);
    const int blocks = c.n * first.per_particle;
    if (save) thin_gate_up_kernel<T, ACT, true, JB><<<blocks, kThinBlock, 0, c.stream>>>(c.s, first, in<T>(x), c.gate, c.up, h, g, u);
    else thin_gate_up_kernel<T, ACT, false, JB><<<blocks, kThinBlock, 0, c.stream>>>(c.s, first, in<T>(x), c.gate, c.up, h, nullptr, nullptr);
    if (const int rc = launched()) return rc;
    thin_down_kernel<T, JB><<<c.n * second.per_particle, kThinBlock, 0, c.stream>>>(c.s, second, h, c.down, out<T>(y));
    return launched();
}

template <class T, int ACT, int JB>
int thin_backward(const FfnCall &c, const svgd_rows &dy, const float *g, const float *u, const svgd_rows &dx, float *dg, float *du)
{
    const ThinGrid hidden(c.s.hidden, 32), input(c.s.width, 32);
    thin_hidden_grad_kernel<T, ACT, JB><<<c.n * hidden.per_particle, kThinBlock, 0, c.stream>>>(c.s, hidden, in<T>(dy), c.down, g, u, dg, du);
    const int rc = launched();
    if (rc || !dx.data) return rc;
    thin_input_grad_kernel<T, JB><<<c.n * input.per_particle, kThinBlock, 0, c.stream>>>(c.s, input, dg, du, c.gate, c.up, out<T>(dx));
    return launched();
}

template <class T, int ACT> int forward_as(const FfnCall &c, const svgd_rows &x, const svgd_rows &y, float *buffer, bool save, float *scratch)
{
    const int64_t plane = c.n * c.s.rows * c.s.hidden_ld;
    float *const h = buffer, *const g = buffer + plane, *const u = buffer + 2 * plane;
    if (thin_forward_rows(c.n, c.s.rows, c.s.hidden))
        return c.s.rows <= 16   ? thin_forward<T, ACT, 1>(c, x, y, h, g, u, save)
               : c.s.rows <= 32 ? thin_forward<T, ACT, 2>(c, x, y, h, g, u, save)
                                : thin_forward<T, ACT, 4>(c, x, y, h, g, u, save);
    const ForwardPlan plan(c.n, c.s.rows, c.s.width, c.s.hidden);
    int rc = with_tile(plan.gate_up.kind, [&](auto tile) {
        using TL = decltype(tile);
        const TileGrid grid(c.n, tiles(c.s.hidden, TL::kI / 2), tiles(c.s.rows, TL::kJ), c.s.width, 1);
        if (grid.total < 0) return (int)SVGD_ERR_TOO_LARGE;
        if (save) gate_up_kernel<TL, T, ACT, true><<<grid.blocks(), TL::kThreads, 0, c.stream>>>(c.s, grid, in<T>(x), c.gate, c.up, h, g, u);
        else gate_up_kernel<TL, T, ACT, false><<<grid.blocks(), TL::kThreads, 0, c.stream>>>(c.s, grid, in<T>(x), c.gate, c.up, h, nullptr, nullptr);
        return launched();
    });
    if (rc) return rc;
    rc = with_tile(plan.down.kind, [&](auto tile) {
        using TL = decltype(tile);
        const TileGrid grid(c.n, tiles(c.s.width, TL::kI), tiles(c.s.rows, TL::kJ), c.s.hidden, plan.down.parts);
        if (grid.total < 0) return (int)SVGD_ERR_TOO_LARGE;
        down_kernel<TL, T><<<grid.blocks(), TL::kThreads, 0, c.stream>>>(c.s, grid, h, c.down, out<T>(y), scratch);
        return launched();
    });
    if (rc || plan.down.parts == 1) return rc;
    return reduce_rows<T>(c, scratch, plan.down.parts, out<T>(y));
}

template <class T, int ACT>
int backward_as(const FfnCall &c, const svgd_rows &dy, const svgd_rows &x, const float *saved, const svgd_rows &dx, const Params &dgate, const Params &dup,
             const Params &ddown, bool accumulate, float *scratch)
{
    const int64_t plane = c.n * c.s.rows * c.s.hidden_ld;
    const float *const h = saved, *const g = saved + plane, *const u = saved + 2 * plane;
    const BackwardPlan plan(c.n, c.s.rows, c.s.width, c.s.hidden);
    float *const dg = scratch, *const du = dg + plan.hidden_floats, *const dx_partial = du + plan.hidden_floats;
    float *const gate_partial = dx_partial + aligned4(plan.input_floats), *const down_partial = gate_partial + aligned4(plan.gate_floats);
    const int gates = (dgate.p ? 1 : 0) + (dup.p ? 1 : 0);
    const bool thin = c.s.rows <= kThinRows;
    if (thin && c.s.rows > 0 && (dx.data || gates)) {
        if (const int rc = c.s.rows <= 16 ? thin_backward<T, ACT, 1>(c, dy, g, u, dx, dg, du) : thin_backward<T, ACT, 2>(c, dy, g, u, dx, dg, du)) return rc;
    }
    if (!thin && (dx.data || gates)) {
        const int rc = with_tile(plan.hidden.kind, [&](auto tile) {
            using TL = decltype(tile);
            const TileGrid grid(c.n, tiles(c.s.hidden, TL::kI), tiles(c.s.rows, TL::kJ), c.s.width, 1);
            if (grid.total < 0) return (int)SVGD_ERR_TOO_LARGE;
            hidden_grad_kernel<TL, T, ACT><<<grid.blocks(), TL::kThreads, 0, c.stream>>>(c.s, grid, in<T>(dy), c.down, g, u, dg, du);
            return launched();
        });
        if (rc) return rc;
    }
    const bool input = !thin && dx.data;
    if (!input && !gates && !ddown.p) return SVGD_OK;
    int rc = with_tile(plan.gradients, [&](auto tile) {
        using TL = decltype(tile);
        const int64_t particle = c.s.rows * c.s.hidden_ld, row = c.s.hidden_ld;
        const int high = (int)tiles(c.s.hidden, TL::kJ);
        const int64_t wide = tiles(c.s.width, TL::kI);
        TileGrid input_grid;
        if (input) {
            const int parts = plan.input_parts;
            input_grid = TileGrid(c.n, wide, tiles(c.s.rows, TL::kJ), c.s.hidden, parts);
            if (parts > 1) input_grid.per = ((c.s.hidden + parts / 2 - 1) / (parts / 2) + kTileK - 1) / kTileK * kTileK; // half of the parts for either half
        }
        WeightGrad<T, float> of_gates{}, of_down{};
        const Rows<const float> dgs{dg, particle, row}, dus{du, particle, row}, hs{h, particle, row};
        if (gates)
            of_gates = {TileGrid(c.n, wide, (int64_t)high * gates, c.s.rows, plan.param_parts), c.s.width, c.s.hidden, high, gates, in<T>(x),
                        {dgate.p ? dgs : dus, dus}, {dgate.p ? dgate : dup, dup}, gate_partial};
        if (ddown.p)
            of_down = {TileGrid(c.n, wide, high, c.s.rows, plan.param_parts), c.s.width, c.s.hidden, high, 1, in<T>(dy), {hs, hs}, {ddown, ddown}, down_partial};
        if (input_grid.total < 0 || of_gates.grid.total < 0 || of_down.grid.total < 0) return (int)SVGD_ERR_TOO_LARGE;
        gradients_kernel<TL, T><<<input_grid.blocks() + of_gates.grid.blocks() + of_down.grid.blocks(), TL::kThreads, 0, c.stream>>>(
            c.s, input_grid, dg, du, c.gate, c.up, out<T>(dx), dx_partial, of_gates, of_down, accumulate);
        return launched();
    });
    if (rc) return rc;
    if (input && plan.input_parts > 1 && (rc = reduce_rows<T>(c, dx_partial, plan.input_parts, out<T>(dx)))) return rc;
    const int64_t size = c.s.width * c.s.hidden;
    if (gates && plan.param_parts > 1) {
        reduce_params_kernel<<<(unsigned)tiles(c.n * gates * size, 256), 256, 0, c.stream>>>(c.n, size, gates, gate_partial, plan.param_parts,
                                                                                            dgate.p ? dgate : dup, dup, accumulate);
        if ((rc = launched())) return rc;
    }
    if (ddown.p && plan.param_parts > 1) {
        reduce_params_kernel<<<(unsigned)tiles(c.n * size, 256), 256, 0, c.stream>>>(c.n, size, 1, down_partial, plan.param_parts, ddown, ddown, accumulate);
        rc = launched();
    }
    return rc;
}

template <class T> int ffn_forward(const FfnCall &c, const svgd_rows &x, const svgd_rows &y, float *buffer, bool save, float *scratch)
{
    return c.activation == SVGD_SILU ? forward_as<T, SVGD_SILU>(c, x, y, buffer, save, scratch) : forward_as<T, SVGD_GELU>(c, x, y, buffer, save, scratch);
}

template <class T>
int ffn_backward(const FfnCall &c, const svgd_rows &dy, const svgd_rows &x, const float *saved, const svgd_rows &dx, const Params &dgate, const Params &dup,
                 const Params &ddown, bool accumulate, float *scratch)
{
    return c.activation == SVGD_SILU ? backward_as<T, SVGD_SILU>(c, dy, x, saved, dx, dgate, dup, ddown, accumulate, scratch)
                                     : backward_as<T, SVGD_GELU>(c, dy, x, saved, dx, dgate, dup, ddown, accumulate, scratch);
}

#ifndef SVGD_FFN_TYPE
extern template int ffn_forward<float>(const FfnCall &, const svgd_rows &, const svgd_rows &, float *, bool, float *);
extern template int ffn_forward<bf16_t>(const FfnCall &, const svgd_rows &, const svgd_rows &, float *, bool, float *);
extern template int ffn_forward<f16_t>(const FfnCall &, const svgd_rows &, const svgd_rows &, float *, bool, float *);
extern template int ffn_backward<float>(const FfnCall &, const svgd_rows &, const svgd_rows &, const float *, const svgd_rows &, const Params &,
                                        const Params &, const Params &, bool, float *);
extern template int ffn_backward<bf16_t>(const FfnCall &, const svgd_rows &, const svgd_rows &, const float *, const svgd_rows &, const Params &,
                                         const Params &, const Params &, bool, float *);
extern template int ffn_backward<f16_t>(const FfnCall &, const svgd_rows &, const svgd_rows &, const float *, const svgd_rows &, const Params &,
                                        const Params &, const Params &, bool, float *);
#endif

} // namespace svgd
