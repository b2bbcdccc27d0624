// The linear maps' launches of one type.
#define SVGD_FFN_TYPE
#include "linear_launch.hpp"

namespace svgd {

template <class T, int JB> static int thin_linear(const LinearCall &c, const LinearOut<T> &to)
{
    const ThinGrid grid(c.s.out, 16);
    thin_linear_kernel<T, JB><<<c.s.n * grid.per_particle, kThinBlock, 0, c.stream>>>(c.s, grid, in<T>(c.x), c.weight, to);
    return launched();
}

template <> int linear_forward<SVGD_LINEAR_TYPE>(const LinearCall &c, const LinearForwardPlan &plan)
{
    typedef SVGD_LINEAR_TYPE T;
    const LinearOut<T> to{c.bias, in<T>(c.residual), out<T>(c.y), c.z};
    if (plan.thin) return c.s.rows <= 16 ? thin_linear<T, 1>(c, to) : thin_linear<T, 2>(c, to);
    const int rc = with_tile(plan.tile.kind, [&](auto tile) {
        using TL = decltype(tile);
        const TileGrid grid(c.s.n, tiles(c.s.out, TL::kI), tiles(c.s.rows, TL::kJ), c.s.width, plan.tile.parts);
        linear_forward_kernel<TL, T><<<grid.blocks(), TL::kThreads, 0, c.stream>>>(c.s, grid, in<T>(c.x), c.weight, to, c.scratch);
        return launched();
    });
    if (rc || plan.tile.parts == 1) return rc;
    linear_join_kernel<T><<<(unsigned)tiles(c.s.n * c.s.rows * c.s.out_ld / 4, 256), 256, 0, c.stream>>>(c.s, c.scratch, plan.tile.parts, to);
    return launched();
}

template <class T, class TD> static int linear_gradients(const LinearCall &c, const LinearBackwardPlan &plan, const Rows<const TD> &dz, float *dx_partial, float *param_partial)
{
    int rc = with_tile(plan.kind, [&](auto tile) {
        using TL = decltype(tile);
        const int64_t wide = tiles(c.s.width, TL::kI);
        const int high = (int)tiles(c.s.out, TL::kJ);
        TileGrid input;
        if (c.dx.data && c.s.rows > 0) input = TileGrid(c.s.n, wide, tiles(c.s.rows, TL::kJ), c.s.out, plan.input_parts);
        WeightGrad<T, TD> grad{};
        if (c.dweight.p) grad = {TileGrid(c.s.n, wide, high, c.s.rows, plan.param_parts), c.s.width, c.s.out, high, 1, in<T>(c.x), {dz, dz}, {c.dweight, c.dweight}, param_partial};
        linear_gradients_kernel<TL, T, TD><<<input.blocks() + grad.grid.blocks(), TL::kThreads, 0, c.stream>>>(c.s, input, dz, c.weight, out<T>(c.dx), dx_partial, grad, c.accumulate);
        return launched();
    });
    if (rc) return rc;
    if (c.dx.data && c.s.rows > 0 && plan.input_parts > 1) {
        const FfnShape s{c.s.n, c.s.rows, c.s.width, c.s.out, c.s.out_ld, c.s.width_ld};
        reduce_rows_kernel<T><<<(unsigned)tiles(c.s.n * c.s.rows * c.s.width_ld / 4, 256), 256, 0, c.stream>>>(s, dx_partial, plan.input_parts, out<T>(c.dx));
        rc = launched();
    }
    return rc;
}

template <> int linear_backward<SVGD_LINEAR_TYPE>(const LinearCall &c, const LinearBackwardPlan &plan)
{
    typedef SVGD_LINEAR_TYPE T;
    float *const dz = c.scratch, *const dx_partial = dz + plan.dz_floats, *const param_partial = dx_partial + aligned4(plan.input_floats), *const sums = param_partial + aligned4(plan.param_floats);
    const bool act = c.s.activation != SVGD_NO_ACTIVATION, products = (c.dx.data && c.s.rows > 0) || c.dweight.p;
    if (c.s.rows > 0 && ((act && products) || c.dbias.p)) {
        const int groups = (int)tiles(c.s.out, 256);
        const int blocks = c.s.n * plan.sums * groups;
        if (act) linear_slope_kernel<T, true><<<blocks, 256, 0, c.stream>>>(c.s, plan.sum_rows, plan.sums, groups, in<T>(c.dy), c.z, products ? dz : nullptr, sums, c.dbias, c.accumulate);
        else linear_slope_kernel<T, false><<<blocks, 256, 0, c.stream>>>(c.s, plan.sum_rows, plan.sums, groups, in<T>(c.dy), nullptr, nullptr, sums, c.dbias, c.accumulate);
        if (const int rc = launched()) return rc;
    }
    const bool all = products && !(c.s.rows == 0 && c.accumulate);
    if (all) {
        const Rows<const float> d = act ? Rows<const float>{dz, c.s.rows * c.s.out_ld, c.s.out_ld} : Rows<const float>{(const float *)c.dy.data, c.dy.particle_stride, c.dy.row_stride};
        const int rc = act || std::is_same<T, float>::value ? linear_gradients<T, float>(c, plan, d, dx_partial, param_partial) : linear_gradients<T, T>(c, plan, in<T>(c.dy), dx_partial, param_partial);
        if (rc) return rc;
    }
    PartSums weight{}, bias{};
    if (all && c.dweight.p && plan.param_parts > 1) weight = {param_partial, plan.param_parts, c.s.width * c.s.out, c.dweight};
    if (c.dbias.p && (plan.sums > 1 || (c.s.rows == 0 && !c.accumulate))) bias = {sums, plan.sums, c.s.out, c.dbias}; // (the sum over no rows is 0)
    if (weight.blocks() + bias.blocks() == 0) return SVGD_OK;
    linear_sums_kernel<<<dim3((unsigned)(weight.blocks() + bias.blocks()), c.s.n), 256, 0, c.stream>>>(weight, bias, c.accumulate);
    return launched();
}

} // namespace svgd
