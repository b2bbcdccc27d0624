// The launches of both passes, by the plan that ffn_rules.hpp makes.  The kernels' instances are compiled type by type (layers_ffn_*.hip).
#pragma once
#include "ffn_thin_kernels.hpp"

namespace svgd {

typedef Tile<4, 8> LargeTile;
typedef Tile<2, 4> SmallTile;
typedef Tile<1, 2> TinyTile;
template <class TL> constexpr bool is_kind(TileKind kind) { return kKinds[kind].i == TL::kI && kKinds[kind].j == TL::kJ && kKinds[kind].threads == TL::kThreads; }
static_assert(is_kind<LargeTile>(kLarge) && is_kind<SmallTile>(kSmall) && is_kind<TinyTile>(kTiny), "the rules reckon with these tiles");

template <class F> int with_tile(TileKind kind, F f)
{
    return kind == kLarge ? f(LargeTile{}) : kind == kSmall ? f(SmallTile{}) : f(TinyTile{});
}

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
int thin_backward(const FfnCall &c, const svgd_rows &dy, const float *g, const float *u, const svgd_rows &dx, bool with_dx, float *dg, float *du)
{
    const ThinGrid hidden(c.s.hidden, 32), input(c.s.width, 32);
    thin_hidden_grad_kernel<T, ACT, JB><<<c.n * hidden.per_particle, kThinBlock, 0, c.stream>>>(c.s, hidden, in<T>(dy), c.down, g, u, dg, du);
    const int rc = launched();
    if (rc || !with_dx) return rc;
    thin_input_grad_kernel<T, JB><<<c.n * input.per_particle, kThinBlock, 0, c.stream>>>(c.s, input, dg, du, c.gate, c.up, out<T>(dx));
    return launched();
}

template <class T, int ACT> int forward_as(const FfnCall &c, const ForwardPlan &plan, const svgd_rows &x, const svgd_rows &y, float *buffer, bool save, float *scratch)
{
    const int64_t plane = c.n * c.s.rows * c.s.hidden_ld;
    float *const h = buffer, *const g = buffer + plane, *const u = buffer + 2 * plane;
    if (plan.thin)
        return c.s.rows <= 16   ? thin_forward<T, ACT, 1>(c, x, y, h, g, u, save)
               : c.s.rows <= 32 ? thin_forward<T, ACT, 2>(c, x, y, h, g, u, save)
                                : thin_forward<T, ACT, 4>(c, x, y, h, g, u, save);
    int rc = with_tile(plan.gate_up.kind, [&](auto tile) {
        using TL = decltype(tile);
        const TileGrid grid(c.n, tiles(c.s.hidden, TL::kI / 2), tiles(c.s.rows, TL::kJ), c.s.width, 1);
        if (save) gate_up_kernel<TL, T, ACT, true><<<grid.blocks(), TL::kThreads, 0, c.stream>>>(c.s, grid, in<T>(x), c.gate, c.up, h, g, u);
        else gate_up_kernel<TL, T, ACT, false><<<grid.blocks(), TL::kThreads, 0, c.stream>>>(c.s, grid, in<T>(x), c.gate, c.up, h, nullptr, nullptr);
        return launched();
    });
    if (rc) return rc;
    rc = with_tile(plan.down.kind, [&](auto tile) {
        using TL = decltype(tile);
        const TileGrid grid(c.n, tiles(c.s.width, TL::kI), tiles(c.s.rows, TL::kJ), c.s.hidden, plan.down.parts);
        down_kernel<TL, T><<<grid.blocks(), TL::kThreads, 0, c.stream>>>(c.s, grid, h, c.down, out<T>(y), scratch);
        return launched();
    });
    if (rc || plan.down.parts == 1) return rc;
    return reduce_rows<T>(c, scratch, plan.down.parts, out<T>(y));
}

template <class T, int ACT>
int backward_as(const FfnCall &c, const BackwardPlan &plan, const svgd_rows &dy, const svgd_rows &x, const float *saved, const svgd_rows &dx, const Params &dgate, const Params &dup,
             const Params &ddown, bool accumulate, float *scratch)
{
    const int64_t plane = c.n * c.s.rows * c.s.hidden_ld;
    const float *const h = saved, *const g = saved + plane, *const u = saved + 2 * plane;
    float *const dg = scratch, *const du = dg + plan.hidden_floats, *const dx_partial = du + plan.hidden_floats;
    float *const gate_partial = dx_partial + aligned4(plan.input_floats), *const down_partial = gate_partial + aligned4(plan.gate_floats);
    const int gates = (dgate.p ? 1 : 0) + (dup.p ? 1 : 0);
    const bool thin = plan.thin;
    if (thin && c.s.rows > 0 && (dx.data || gates)) {
        const bool with_dx = plan.thin_input && dx.data;
        if (const int rc = c.s.rows <= 16 ? thin_backward<T, ACT, 1>(c, dy, g, u, dx, with_dx, dg, du) : thin_backward<T, ACT, 2>(c, dy, g, u, dx, with_dx, dg, du)) return rc;
    }
    if (!thin && (dx.data || gates)) {
        const int rc = with_tile(plan.hidden.kind, [&](auto tile) {
            using TL = decltype(tile);
            const TileGrid grid(c.n, tiles(c.s.hidden, TL::kI), tiles(c.s.rows, TL::kJ), c.s.width, 1);
            hidden_grad_kernel<TL, T, ACT><<<grid.blocks(), TL::kThreads, 0, c.stream>>>(c.s, grid, in<T>(dy), c.down, g, u, dg, du);
            return launched();
        });
        if (rc) return rc;
    }
    const bool input = !plan.thin_input && dx.data;
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

template <class T> int ffn_forward(const FfnCall &c, const ForwardPlan &plan, const svgd_rows &x, const svgd_rows &y, float *buffer, bool save, float *scratch)
{
    return c.activation == SVGD_SILU ? forward_as<T, SVGD_SILU>(c, plan, x, y, buffer, save, scratch) : forward_as<T, SVGD_GELU>(c, plan, x, y, buffer, save, scratch);
}

template <class T>
int ffn_backward(const FfnCall &c, const BackwardPlan &plan, const svgd_rows &dy, const svgd_rows &x, const float *saved, const svgd_rows &dx, const Params &dgate, const Params &dup,
                 const Params &ddown, bool accumulate, float *scratch)
{
    return c.activation == SVGD_SILU ? backward_as<T, SVGD_SILU>(c, plan, dy, x, saved, dx, dgate, dup, ddown, accumulate, scratch)
                                     : backward_as<T, SVGD_GELU>(c, plan, dy, x, saved, dx, dgate, dup, ddown, accumulate, scratch);
}

#ifndef SVGD_FFN_TYPE
extern template int ffn_forward<float>(const FfnCall &, const ForwardPlan &, const svgd_rows &, const svgd_rows &, float *, bool, float *);
extern template int ffn_forward<bf16_t>(const FfnCall &, const ForwardPlan &, const svgd_rows &, const svgd_rows &, float *, bool, float *);
extern template int ffn_forward<f16_t>(const FfnCall &, const ForwardPlan &, const svgd_rows &, const svgd_rows &, float *, bool, float *);
extern template int ffn_backward<float>(const FfnCall &, const BackwardPlan &, const svgd_rows &, const svgd_rows &, const float *, const svgd_rows &, const Params &,
                                        const Params &, const Params &, bool, float *);
extern template int ffn_backward<bf16_t>(const FfnCall &, const BackwardPlan &, const svgd_rows &, const svgd_rows &, const float *, const svgd_rows &, const Params &,
                                         const Params &, const Params &, bool, float *);
extern template int ffn_backward<f16_t>(const FfnCall &, const BackwardPlan &, const svgd_rows &, const svgd_rows &, const float *, const svgd_rows &, const Params &,
                                        const Params &, const Params &, bool, float *);
#endif

} // namespace svgd
