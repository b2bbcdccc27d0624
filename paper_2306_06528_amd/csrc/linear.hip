// Host side of the linear maps (include/svgd_attention.h): checks of arguments.
#include "linear_launch.hpp"

using namespace svgd;

namespace {

bool sized(int n, int64_t rows, int64_t width, int64_t out)
{
    return n >= 1 && n <= SVGD_MAX_PARTICLES && rows >= 0 && rows <= SVGD_LAYER_MAX_ROWS && width >= 1 && width <= SVGD_LAYER_MAX_WIDTH && out >= 1 && out <= SVGD_LAYER_MAX_WIDTH;
}
template <class F> int for_type(int dtype, F f) { return dtype == SVGD_F32 ? f(float{}) : dtype == SVGD_BF16 ? f(bf16_t{}) : f(f16_t{}); }

int check(int dtype, int activation, int n, int64_t rows, int64_t width, int64_t out, const svgd_rows &x, const Params &weight)
{
    if (const int rc = check_sizes(dtype, n, rows, width, SVGD_LAYER_MAX_WIDTH)) return rc;
    if (out < 1 || activation < SVGD_SILU || activation > SVGD_NO_ACTIVATION) return SVGD_ERR_INVALID_ARG;
    if (out > SVGD_LAYER_MAX_WIDTH) return SVGD_ERR_TOO_LARGE;
    if ((rows > 0 && !valid_input(x, dtype, rows)) || !valid_params(weight, n, false)) return SVGD_ERR_INVALID_ARG;
    return SVGD_OK;
}
int64_t size_of(int64_t width, int64_t out) { return width > 0 && out > 0 && width <= SVGD_LAYER_MAX_WIDTH && out <= SVGD_LAYER_MAX_WIDTH ? width * out : 0; }

} // namespace

extern "C" {

size_t svgd_linear_saved(int n, int64_t rows, int64_t out)
{
    if (!sized(n, rows, 1, out)) return 0;
    return (size_t)n * rows * linear_ld(out) * 4;
}

size_t svgd_linear_forward_scratch(int n, int64_t rows, int64_t width, int64_t out)
{
    if (!sized(n, rows, width, out) || rows == 0) return 0;
    return LinearForwardPlan(n, rows, width, out).scratch(n, rows, out);
}

int svgd_linear_forward(int dtype, int activation, int n, int64_t rows, int64_t width, int64_t out, svgd_rows x, const float *weight, int64_t weight_stride, const float *bias,
                        int64_t bias_stride, svgd_rows residual, svgd_rows y, void *z, size_t z_bytes, void *scratch, size_t scratch_bytes, void *stream)
{
    const int64_t size = size_of(width, out);
    LinearCall c{};
    c.s = {n, activation, rows, width, out, linear_ld(out), linear_ld(width)};
    c.weight = {weight, weight_stride, size};
    c.bias = {bias, bias_stride, out};
    if (const int rc = check(dtype, activation, n, rows, width, out, x, c.weight)) return rc;
    if (bias && !valid_params(c.bias, n, false)) return SVGD_ERR_INVALID_ARG;
    if (rows == 0) return SVGD_OK;
    const LinearForwardPlan plan(n, rows, width, out);
    const size_t z_need = z ? svgd_linear_saved(n, rows, out) : 0, need = plan.scratch(n, rows, out);
    if (!valid_output(y, dtype, n, rows, out) || (residual.data && !valid_input(residual, dtype, rows)) || !aligned_to(z, 16) || z_bytes < z_need ||
        (need && (!scratch || !aligned_to(scratch, 16) || scratch_bytes < need)))
        return SVGD_ERR_INVALID_ARG;
    const Extent written[3] = {extent(y, dtype, n, rows, out), extent(z, z_need), extent(scratch, need)};
    const Extent read[4] = {extent(x, dtype, n, rows, width), extent(weight, weight_stride, n, size), bias ? extent(bias, bias_stride, n, out) : Extent{0, 0},
                            residual.data ? extent(residual, dtype, n, rows, out) : Extent{0, 0}};
    for (int i = 0; i < 3; ++i) {
        for (int r = 0; r < 4; ++r)
            if (written[i].meets(read[r])) return SVGD_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (written[i].meets(written[j])) return SVGD_ERR_INVALID_ARG;
    }
    if (!plan.fits()) return SVGD_ERR_TOO_LARGE;
    c.x = x;
    c.y = y;
    c.residual = residual;
    c.z = (float *)z;
    c.scratch = (float *)scratch;
    c.stream = (hipStream_t)stream;
    return for_type(dtype, [&](auto t) { return linear_forward<decltype(t)>(c, plan); });
}

size_t svgd_linear_scratch(int n, int64_t rows, int64_t width, int64_t out)
{
    if (!sized(n, rows, width, out)) return 0;
    return LinearBackwardPlan(n, rows, width, out).scratch();
}

int svgd_linear_backward(int dtype, int activation, int n, int64_t rows, int64_t width, int64_t out, svgd_rows dy, svgd_rows x, const float *weight, int64_t weight_stride,
                         const void *z, size_t z_bytes, svgd_rows dx, float *dweight, int64_t dweight_stride, float *dbias, int64_t dbias_stride, int accumulate, void *scratch,
                         size_t scratch_bytes, void *stream)
{
    const int64_t size = size_of(width, out);
    LinearCall c{};
    c.s = {n, activation, rows, width, out, linear_ld(out), linear_ld(width)};
    c.weight = {weight, weight_stride, size};
    c.dweight = {dweight, dweight_stride, size};
    c.dbias = {dbias, dbias_stride, out};
    if (const int rc = check(dtype, activation, n, rows, width, out, x, c.weight)) return rc;
    for (const Params *g : {&c.dweight, &c.dbias})
        if (g->p && (!valid_params(*g, n, true) || params_meet(*g, c.weight, n))) return SVGD_ERR_INVALID_ARG;
    if (dweight && dbias && params_meet(c.dweight, c.dbias, n)) return SVGD_ERR_INVALID_ARG;
    const bool act = activation != SVGD_NO_ACTIVATION;
    const LinearBackwardPlan plan(n, rows, width, out, act);
    if (rows > 0) {
        const size_t z_need = act ? svgd_linear_saved(n, rows, out) : 0, need = plan.scratch();
        if (!valid_input(dy, dtype, rows) || (act && (!z || !aligned_to(z, 16) || z_bytes < z_need)) || (dx.data && !valid_output(dx, dtype, n, rows, width)) || !scratch ||
            !aligned_to(scratch, 16) || scratch_bytes < need)
            return SVGD_ERR_INVALID_ARG;
        const Extent written[4] = {extent(scratch, need), dx.data ? extent(dx, dtype, n, rows, width) : Extent{0, 0}, dweight ? extent(dweight, dweight_stride, n, size) : Extent{0, 0},
                                   dbias ? extent(dbias, dbias_stride, n, out) : Extent{0, 0}};
        const Extent read[4] = {extent(dy, dtype, n, rows, out), extent(x, dtype, n, rows, width), extent(z, z_need), extent(weight, weight_stride, n, size)};
        for (int i = 0; i < 4; ++i) {
            for (int r = 0; r < (i < 2 ? 4 : 3); ++r) // (the gradients may lie between the weights, in the same rows: looked at above)
                if (written[i].meets(read[r])) return SVGD_ERR_INVALID_ARG;
            for (int j = 0; j < i && j < 2; ++j)
                if (written[i].meets(written[j])) return SVGD_ERR_INVALID_ARG;
        }
    }
    if (!plan.fits()) return SVGD_ERR_TOO_LARGE;
    c.x = x;
    c.dy = dy;
    c.dx = dx;
    c.z = (float *)const_cast<void *>(z);
    c.scratch = (float *)scratch;
    c.accumulate = accumulate != 0;
    c.stream = (hipStream_t)stream;
    return for_type(dtype, [&](auto t) { return linear_backward<decltype(t)>(c, plan); });
}

} // extern "C"
