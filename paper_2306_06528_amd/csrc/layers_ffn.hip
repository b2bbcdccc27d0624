// Host side of the gated feed-forward block (include/svgd_layers.h): checks and launches.
#include "ffn_thin_kernels.hpp"

using namespace svgd;

namespace {

int64_t hidden_ld(int64_t hidden) { return (hidden + 31) / 32 * 32; } // rows of the buffers start on 128 bytes

bool sized(int n, int64_t rows, int64_t width, int64_t hidden)
{
    return n >= 1 && n <= SVGD_MAX_PARTICLES && rows >= 0 && rows <= SVGD_LAYER_MAX_ROWS && width >= 1 && width <= SVGD_LAYER_MAX_WIDTH &&
           hidden >= 1 && hidden <= SVGD_LAYER_MAX_WIDTH;
}

int64_t tiles(int64_t size, int tile) { return (size + tile - 1) / tile; }

struct Call {
    int dtype, activation, n;
    FfnShape s;
    Params gate, up, down;
    hipStream_t stream;
};

template <class T> Rows<const T> in(const svgd_rows &r) { return {(const T *)r.data, r.particle_stride, r.row_stride}; }
template <class T> Rows<T> out(const svgd_rows &r) { return {(T *)r.data, r.particle_stride, r.row_stride}; }
int launched() { return hipGetLastError() == hipSuccess ? SVGD_OK : SVGD_ERR_DEVICE; }

// Up to so many rows per particle the weights go straight from memory to the matrix cores (ffn_thin_kernels.hpp).
constexpr int64_t kThinRows = 32;

template <class T, int ACT, int JB> int thin_forward(const Call &c, const svgd_rows &x, const svgd_rows &y, float *h, float *g, float *u, bool save)
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
int thin_backward(const Call &c, const svgd_rows &dy, const float *g, const float *u, const svgd_rows &dx, float *dg, float *du)
{
    const ThinGrid hidden(c.s.hidden, 32), input(c.s.width, 32);
    thin_hidden_grad_kernel<T, ACT, JB><<<c.n * hidden.per_particle, kThinBlock, 0, c.stream>>>(c.s, hidden, in<T>(dy), c.down, g, u, dg, du);
    const int rc = launched();
    if (rc || !dx.data) return rc;
    thin_input_grad_kernel<T, JB><<<c.n * input.per_particle, kThinBlock, 0, c.stream>>>(c.s, input, dg, du, c.gate, c.up, out<T>(dx));
    return launched();
}

template <class T, int ACT> int forward(const Call &c, const svgd_rows &x, const svgd_rows &y, float *buffer, bool save)
{
    const int64_t plane = c.n * c.s.rows * c.s.hidden_ld;
    float *const h = buffer, *const g = buffer + plane, *const u = buffer + 2 * plane;
    if (c.s.rows <= kThinRows)
        return c.s.rows <= 16 ? thin_forward<T, ACT, 1>(c, x, y, h, g, u, save) : thin_forward<T, ACT, 2>(c, x, y, h, g, u, save);
    typedef Tile<4, 8> TL;
    const TileGrid first(c.n, tiles(c.s.hidden, TL::kI / 2), tiles(c.s.rows, TL::kJ)), second(c.n, tiles(c.s.width, TL::kI), tiles(c.s.rows, TL::kJ));
    if (first.total < 0 || second.total < 0) return SVGD_ERR_TOO_LARGE;
    if (save) gate_up_kernel<TL, T, ACT, true><<<first.blocks(), TL::kThreads, 0, c.stream>>>(c.s, first, in<T>(x), c.gate, c.up, h, g, u);
    else gate_up_kernel<TL, T, ACT, false><<<first.blocks(), TL::kThreads, 0, c.stream>>>(c.s, first, in<T>(x), c.gate, c.up, h, nullptr, nullptr);
    if (const int rc = launched()) return rc;
    down_kernel<TL, T><<<second.blocks(), TL::kThreads, 0, c.stream>>>(c.s, second, h, c.down, out<T>(y));
    return launched();
}

template <class T, int ACT>
int backward(const Call &c, const svgd_rows &dy, const svgd_rows &x, const float *saved, const svgd_rows &dx, const Params &dgate, const Params &dup,
             const Params &ddown, bool accumulate, float *scratch)
{
    const int64_t plane = c.n * c.s.rows * c.s.hidden_ld;
    const float *const h = saved, *const g = saved + plane, *const u = saved + 2 * plane;
    float *const dg = scratch, *const du = scratch + plane;
    typedef Tile<4, 8> TL;
    const int64_t tj = tiles(c.s.rows, TL::kJ);
    const TileGrid hidden(c.n, tiles(c.s.hidden, TL::kI), tj), input(c.n, tiles(c.s.width, TL::kI), tj);
    const int gates = (dgate.p ? 1 : 0) + (dup.p ? 1 : 0), high = (int)tiles(c.s.hidden, TL::kJ);
    const TileGrid gate_up(c.n, tiles(c.s.width, TL::kI), (int64_t)high * gates), down(c.n, tiles(c.s.width, TL::kI), high);
    if (hidden.total < 0 || input.total < 0 || gate_up.total < 0 || down.total < 0) return SVGD_ERR_TOO_LARGE;
    const bool thin = c.s.rows <= kThinRows;
    if (thin && c.s.rows > 0 && (dx.data || gates)) {
        if (const int rc = c.s.rows <= 16 ? thin_backward<T, ACT, 1>(c, dy, g, u, dx, dg, du) : thin_backward<T, ACT, 2>(c, dy, g, u, dx, dg, du)) return rc;
    }
    if (!thin && (dx.data || gates)) {
        hidden_grad_kernel<TL, T, ACT><<<hidden.blocks(), TL::kThreads, 0, c.stream>>>(c.s, hidden, in<T>(dy), c.down, g, u, dg, du);
        if (const int rc = launched()) return rc;
    }
    if (!thin && dx.data) {
        input_grad_kernel<TL, T><<<input.blocks(), TL::kThreads, 0, c.stream>>>(c.s, input, dg, du, c.gate, c.up, out<T>(dx));
        if (const int rc = launched()) return rc;
    }
    const int64_t particle = c.s.rows * c.s.hidden_ld, row = c.s.hidden_ld;
    if (gates) {
        const Rows<const float> a{dgate.p ? dg : du, particle, row}, b{du, particle, row};
        weight_grad_kernel<TL, T, float, false><<<gate_up.blocks(), TL::kThreads, 0, c.stream>>>(c.s.rows, c.s.width, c.s.hidden, gate_up, high, in<T>(x), a, b,
                                                                             dgate.p ? dgate : dup, dup, accumulate);
        if (const int rc = launched()) return rc;
    }
    if (ddown.p) {
        const Rows<const float> hs{h, particle, row};
        weight_grad_kernel<TL, T, float, true><<<down.blocks(), TL::kThreads, 0, c.stream>>>(c.s.rows, c.s.width, c.s.hidden, down, high, in<T>(dy), hs, hs,
                                                                                            ddown, ddown, accumulate);
        if (const int rc = launched()) return rc;
    }
    return SVGD_OK;
}

template <class F> int for_type(int dtype, int activation, F f)
{
    const bool silu = activation == SVGD_SILU;
    switch (dtype) {
    case SVGD_F32: return silu ? f(float{}, std::integral_constant<int, SVGD_SILU>{}) : f(float{}, std::integral_constant<int, SVGD_GELU>{});
    case SVGD_BF16: return silu ? f(bf16_t{}, std::integral_constant<int, SVGD_SILU>{}) : f(bf16_t{}, std::integral_constant<int, SVGD_GELU>{});
    default: return silu ? f(f16_t{}, std::integral_constant<int, SVGD_SILU>{}) : f(f16_t{}, std::integral_constant<int, SVGD_GELU>{});
    }
}

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

size_t svgd_gated_ffn_scratch(int n, int64_t rows, int64_t width, int64_t hidden)
{
    if (!sized(n, rows, width, hidden)) return 0;
    return (size_t)n * (size_t)rows * (size_t)hidden_ld(hidden) * 4 * 2;
}

int svgd_gated_ffn_forward(int dtype, int activation, int n, int64_t rows, int64_t width, int64_t hidden, svgd_rows x, const float *gate,
                           int64_t gate_stride, const float *up, int64_t up_stride, const float *down, int64_t down_stride, svgd_rows y, int save,
                           void *buffer, size_t buffer_bytes, void *stream)
{
    const int64_t size = width > 0 && hidden > 0 && width <= SVGD_LAYER_MAX_WIDTH && hidden <= SVGD_LAYER_MAX_WIDTH ? width * hidden : 0;
    const Call c{dtype, activation, n, {rows, width, hidden, hidden_ld(hidden)}, {gate, gate_stride, size}, {up, up_stride, size}, {down, down_stride, size},
                 (hipStream_t)stream};
    if (const int rc = check(dtype, activation, n, rows, width, hidden, x, c.gate, c.up, c.down)) return rc;
    if (rows == 0) return SVGD_OK;
    const size_t need = svgd_gated_ffn_buffer(n, rows, width, hidden, save);
    if (!valid_output(y, dtype, n, rows, width) || !buffer || !aligned_to(buffer, 16) || buffer_bytes < need) return SVGD_ERR_INVALID_ARG;
    const Extent written[2] = {extent(y, dtype, n, rows, width), extent(buffer, need)};
    const Extent read[4] = {extent(x, dtype, n, rows, width), extent(gate, gate_stride, n, size), extent(up, up_stride, n, size),
                            extent(down, down_stride, n, size)};
    if (written[0].meets(written[1])) return SVGD_ERR_INVALID_ARG;
    for (const Extent &w : written)
        for (const Extent &r : read)
            if (w.meets(r)) return SVGD_ERR_INVALID_ARG;
    return for_type(dtype, activation, [&](auto t, auto act) { return forward<decltype(t), decltype(act)::value>(c, x, y, (float *)buffer, save != 0); });
}

int svgd_gated_ffn_backward(int dtype, int activation, int n, int64_t rows, int64_t width, int64_t hidden, svgd_rows dy, svgd_rows x, const float *gate,
                            int64_t gate_stride, const float *up, int64_t up_stride, const float *down, int64_t down_stride, const void *saved,
                            size_t saved_bytes, svgd_rows dx, float *dgate, int64_t dgate_stride, float *dup, int64_t dup_stride, float *ddown,
                            int64_t ddown_stride, int accumulate, void *scratch, size_t scratch_bytes, void *stream)
{
    const int64_t size = width > 0 && hidden > 0 && width <= SVGD_LAYER_MAX_WIDTH && hidden <= SVGD_LAYER_MAX_WIDTH ? width * hidden : 0;
    const Call c{dtype, activation, n, {rows, width, hidden, hidden_ld(hidden)}, {gate, gate_stride, size}, {up, up_stride, size}, {down, down_stride, size},
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
    if (rows > 0) {
        const size_t saved_need = svgd_gated_ffn_buffer(n, rows, width, hidden, 1), need = svgd_gated_ffn_scratch(n, rows, width, hidden);
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
    return for_type(dtype, activation, [&](auto t, auto act) {
        return backward<decltype(t), decltype(act)::value>(c, dy, x, (const float *)saved, dx, grads[0], grads[1], grads[2], accumulate != 0, (float *)scratch);
    });
}

} // extern "C"
