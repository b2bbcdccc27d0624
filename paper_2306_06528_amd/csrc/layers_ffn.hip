// Host side of the gated feed-forward block (include/svgd_layers.h): checks of arguments.
#include "ffn_launch.hpp"

using namespace svgd;

namespace {

bool sized(int n, int64_t rows, int64_t width, int64_t hidden)
{
    return n >= 1 && n <= SVGD_MAX_PARTICLES && rows >= 0 && rows <= SVGD_LAYER_MAX_ROWS && width >= 1 && width <= SVGD_LAYER_MAX_WIDTH &&
           hidden >= 1 && hidden <= SVGD_LAYER_MAX_WIDTH;
}

template <class F> int for_type(int dtype, F f) { return dtype == SVGD_F32 ? f(float{}) : dtype == SVGD_BF16 ? f(bf16_t{}) : f(f16_t{}); }

// Sizes, type, activation, x and the parameters of both passes.
int check(int dtype, int activation, int n, int64_t rows, int64_t width, int64_t hidden, const svgd_rows &x, const Params &gate, const Params &up,
          const Params &down)
{
    int rc = check_sizes(dtype, n, rows, width, SVGD_LAYER_MAX_WIDTH);
    if (rc) return rc;
    if (hidden < 1 || (activation != SVGD_SILU && activation != SVGD_GELU)) return SVGD_ERR_INVALID_ARG;
    if (hidden > SVGD_LAYER_MAX_WIDTH) return SVGD_ERR_TOO_LARGE;
    if ((rows > 0 && !valid_input(x, dtype, rows)) || !valid_params(gate, n, false) || !valid_params(up, n, false) || !valid_params(down, n, false))
        return SVGD_ERR_INVALID_ARG;
    return SVGD_OK;
}

} // namespace

extern "C" {

size_t svgd_gated_ffn_buffer(int n, int64_t rows, int64_t width, int64_t hidden, int save)
{
    if (!sized(n, rows, width, hidden)) return 0;
    return (size_t)n * (size_t)rows * (size_t)hidden_ld(hidden) * 4 * (save ? 3 : 1);
}

size_t svgd_gated_ffn_forward_scratch(int n, int64_t rows, int64_t width, int64_t hidden)
{
    if (!sized(n, rows, width, hidden) || rows == 0) return 0;
    return ForwardPlan(n, rows, width, hidden).scratch(n, rows, width);
}

size_t svgd_gated_ffn_scratch(int n, int64_t rows, int64_t width, int64_t hidden)
{
    if (!sized(n, rows, width, hidden)) return 0;
    const size_t all = BackwardPlan(n, rows, width, hidden, true).scratch(), dx_alone = BackwardPlan(n, rows, width, hidden, false).scratch();
    return all > dx_alone ? all : dx_alone;
}

int svgd_gated_ffn_forward(int dtype, int activation, int n, int64_t rows, int64_t width, int64_t hidden, svgd_rows x, const float *gate,
                           int64_t gate_stride, const float *up, int64_t up_stride, const float *down, int64_t down_stride, svgd_rows y, int save,
                           void *buffer, size_t buffer_bytes, void *scratch, size_t scratch_bytes, void *stream)
{
    const int64_t size = width > 0 && hidden > 0 && width <= SVGD_LAYER_MAX_WIDTH && hidden <= SVGD_LAYER_MAX_WIDTH ? width * hidden : 0;
    const FfnCall c{dtype, activation, n, {n, rows, width, hidden, hidden_ld(hidden), width_ld(width)}, {gate, gate_stride, size}, {up, up_stride, size}, {down, down_stride, size},
                 (hipStream_t)stream};
    if (const int rc = check(dtype, activation, n, rows, width, hidden, x, c.gate, c.up, c.down)) return rc;
    if (rows == 0) return SVGD_OK;
    const size_t need = svgd_gated_ffn_buffer(n, rows, width, hidden, save);
    const ForwardPlan plan(n, rows, width, hidden);
    const size_t scratch_need = plan.scratch(n, rows, width);
    if (!valid_output(y, dtype, n, rows, width) || !buffer || !aligned_to(buffer, 16) || buffer_bytes < need ||
        (scratch_need > 0 && (!scratch || !aligned_to(scratch, 16) || scratch_bytes < scratch_need)))
        return SVGD_ERR_INVALID_ARG;
    const Extent written[3] = {extent(y, dtype, n, rows, width), extent(buffer, need), extent(scratch, scratch_need)};
    const Extent read[4] = {extent(x, dtype, n, rows, width), extent(gate, gate_stride, n, size), extent(up, up_stride, n, size),
                            extent(down, down_stride, n, size)};
    if (written[0].meets(written[1]) || written[0].meets(written[2]) || written[1].meets(written[2])) return SVGD_ERR_INVALID_ARG;
    for (const Extent &w : written)
        for (const Extent &r : read)
            if (w.meets(r)) return SVGD_ERR_INVALID_ARG;
    if (!plan.fits()) return SVGD_ERR_TOO_LARGE;
    return for_type(dtype, [&](auto t) { return ffn_forward<decltype(t)>(c, plan, x, y, (float *)buffer, save != 0, (float *)scratch); });
}

int svgd_gated_ffn_backward(int dtype, int activation, int n, int64_t rows, int64_t width, int64_t hidden, svgd_rows dy, svgd_rows x, const float *gate,
                            int64_t gate_stride, const float *up, int64_t up_stride, const float *down, int64_t down_stride, const void *saved,
                            size_t saved_bytes, svgd_rows dx, float *dgate, int64_t dgate_stride, float *dup, int64_t dup_stride, float *ddown,
                            int64_t ddown_stride, int accumulate, void *scratch, size_t scratch_bytes, void *stream)
{
    const int64_t size = width > 0 && hidden > 0 && width <= SVGD_LAYER_MAX_WIDTH && hidden <= SVGD_LAYER_MAX_WIDTH ? width * hidden : 0;
    const FfnCall c{dtype, activation, n, {n, rows, width, hidden, hidden_ld(hidden), width_ld(width)}, {gate, gate_stride, size}, {up, up_stride, size}, {down, down_stride, size},
                 (hipStream_t)stream};
    if (const int rc = check(dtype, activation, n, rows, width, hidden, x, c.gate, c.up, c.down)) return rc;
    const Params grads[3] = {{dgate, dgate_stride, size}, {dup, dup_stride, size}, {ddown, ddown_stride, size}};
    for (const Params &g : grads) {
        if (!g.p) continue;
        if (!valid_params(g, n, true)) return SVGD_ERR_INVALID_ARG;
        for (const Params *p : {&c.gate, &c.up, &c.down})
            if (params_meet(g, *p, n)) return SVGD_ERR_INVALID_ARG;
        for (const Params &o : grads)
            if (&o > &g && o.p && params_meet(g, o, n)) return SVGD_ERR_INVALID_ARG;
    }
    const BackwardPlan plan(n, rows, width, hidden, grads[0].p || grads[1].p || grads[2].p);
    if (rows > 0) {
        const size_t saved_need = svgd_gated_ffn_buffer(n, rows, width, hidden, 1), need = plan.scratch();
        if (!valid_input(dy, dtype, rows) || !saved || !aligned_to(saved, 16) || saved_bytes < saved_need || !scratch || !aligned_to(scratch, 16) ||
            scratch_bytes < need || (dx.data && !valid_output(dx, dtype, n, rows, width)))
            return SVGD_ERR_INVALID_ARG;
        const Extent acts[3] = {extent(dy, dtype, n, rows, width), extent(x, dtype, n, rows, width), extent(saved, saved_need)};
        const Extent params[3] = {extent(gate, gate_stride, n, size), extent(up, up_stride, n, size), extent(down, down_stride, n, size)};
        const Extent work = extent(scratch, need), dxe = dx.data ? extent(dx, dtype, n, rows, width) : Extent{0, 0};
        if (work.meets(dxe)) return SVGD_ERR_INVALID_ARG;
        for (const Extent &e : acts)
            if (work.meets(e) || dxe.meets(e)) return SVGD_ERR_INVALID_ARG;
        for (const Extent &e : params)
            if (work.meets(e) || dxe.meets(e)) return SVGD_ERR_INVALID_ARG;
        for (const Params &g : grads) {
            if (!g.p) continue;
            const Extent e = extent(g.p, g.stride, n, size);
            if (work.meets(e) || dxe.meets(e) || acts[0].meets(e) || acts[1].meets(e) || acts[2].meets(e)) return SVGD_ERR_INVALID_ARG;
        }
    }
    if (!plan.fits()) return SVGD_ERR_TOO_LARGE;
    return for_type(dtype, [&](auto t) {
        return ffn_backward<decltype(t)>(c, plan, dy, x, (const float *)saved, dx, grads[0], grads[1], grads[2], accumulate != 0, (float *)scratch);
    });
}

} // extern "C"
