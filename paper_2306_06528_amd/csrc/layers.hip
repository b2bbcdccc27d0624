// Host side of layer norm and dropout (include/svgd_layers.h): checks and launches.
#include "dropout_kernels.hpp"
#include "norm_kernels.hpp"

#include <cmath>

using namespace svgd;

namespace {

int launched() { return hipGetLastError() == hipSuccess ? SVGD_OK : SVGD_ERR_DEVICE; }

// The team of threads that holds a row, and how many values each of them.
struct Team {
    int threads, values;
};
Team team_for(int64_t width)
{
    if (width <= 64) return {8, 8};
    if (width <= 128) return {16, 8};
    if (width <= 256) return {32, 8};
    if (width <= 512) return {64, 8};
    if (width <= 1024) return {64, 16};
    if (width <= 2048) return {256, 8};
    if (width <= 4096) return {256, 16};
    if (width <= 8192) return {1024, 8};
    return {1024, 16};
}

template <class F> int for_team(int64_t width, F f)
{
    using std::integral_constant;
    const Team t = team_for(width);
    if (t.threads == 8) return f(integral_constant<int, 8>{}, integral_constant<int, 8>{});
    if (t.threads == 16) return f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
    if (t.threads == 32) return f(integral_constant<int, 32>{}, integral_constant<int, 8>{});
    if (t.threads == 64) return t.values == 8 ? f(integral_constant<int, 64>{}, integral_constant<int, 8>{}) : f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
    if (t.threads == 256) return t.values == 8 ? f(integral_constant<int, 256>{}, integral_constant<int, 8>{}) : f(integral_constant<int, 256>{}, integral_constant<int, 16>{});
    return t.values == 8 ? f(integral_constant<int, 1024>{}, integral_constant<int, 8>{}) : f(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
}

template <class F> int for_type(int dtype, F f)
{
    if (dtype == SVGD_F32) return f(float{});
    if (dtype == SVGD_BF16) return f(bf16_t{});
    return f(f16_t{});
}

// The rows of a particle in at most about `most` / n workgroups, each a multiple of the rows that it has at a time.
NormShape split_rows(int n, int64_t rows, int64_t width, int64_t most)
{
    const Team t = team_for(width);
    const int64_t at_a_time = (t.threads > 256 ? t.threads : 256) / t.threads;
    const int64_t blocks = most / n > 1 ? most / n : 1;
    int64_t per = (rows + blocks - 1) / blocks;
    per = (per + at_a_time - 1) / at_a_time * at_a_time;
    if (per < 1) per = 1;
    return {rows, (int)width, (int)((rows + per - 1) / per), per};
}

// Forward: up to 4,096 workgroups, but beyond 512 two turns for each, so that the second row's load hides behind the first's
// sums (16 x 200 x 64 fp32, 100 turns: 3.0 us one by one, 4.1 two by two).  us at 1,024 / 2,048 / 4,096: 16 x 8,192 x 1,024 bf16 110 / 110 / 104, 8 x 1,576 x 384 bf16 (3,152 turns) 9.1 / 8.2 / 8.8, 5 x 1,003 x 1,001 fp32
// (1,255 turns) 10.0 / 11.9 / 11.8.
NormShape forward_split(int n, int64_t rows, int64_t width)
{
    const Team t = team_for(width);
    const int64_t turns = n * rows * t.threads / (t.threads > 256 ? t.threads : 256);
    return split_rows(n, rows, width, turns / 2 > 4096 ? 4096 : turns / 2 > 512 ? turns / 2 : 512);
}

// Backward: as many workgroups as run at a time, by their registers: four per CU, two with 16 values per thread, one of 1,024
// threads; fewer partial sums are left then.  Activations that the memory-side cache does not hold like one per CU better.
// us at 256 / 512 / 1,024: 8 x 1,576 x 384 bf16 24 / 18 / 15, 5 x 1,003 x 1,001 fp32 19 / 17.5 / 21, 16 x 8,192 x 1,024 bf16 (805 MB)
// 157 / 163 / 171, 8 x 16,384 x 256 bf16 (201 MB) 40 / 34 / 35.  (At four bytes
// per value: their type is not known where scratch memory is asked for.)
NormShape backward_split(int n, int64_t rows, int64_t width)
{
    const Team t = team_for(width);
    const bool big = n * rows * width * 4 > (int64_t)256 << 20;
    return split_rows(n, rows, width, big || t.threads > 256 ? 256 : t.values > 8 ? 512 : 1024);
}

template <class T> ActRows<const T> in(const svgd_rows &r) { return {(const T *)r.data, r.particle_stride, r.row_stride}; }
template <class T> ActRows<T> out(const svgd_rows &r) { return {(T *)r.data, r.particle_stride, r.row_stride}; }

bool flat(const svgd_rows &r, int n, int64_t rows, int64_t width)
{
    return (rows == 1 || r.row_stride == width) && (n == 1 || r.particle_stride == rows * width);
}

bool same_rows(const svgd_rows &a, const svgd_rows &b, int n, int64_t rows)
{
    return a.data == b.data && (n == 1 || a.particle_stride == b.particle_stride) && (rows == 1 || a.row_stride == b.row_stride);
}

} // namespace

extern "C" {

int svgd_layer_norm_forward(int dtype, int n, int64_t rows, int64_t width, svgd_rows x, const float *weight, int64_t weight_stride, const float *bias,
                            int64_t bias_stride, double eps, svgd_rows y, float *mean, float *rstd, void *stream)
{
    if (const int rc = check_sizes(dtype, n, rows, width, SVGD_LAYER_MAX_NORM)) return rc;
    const Params w{weight, weight_stride, width}, b{bias, bias_stride, width};
    if (!std::isfinite(eps) || eps < 0 || !valid_params(w, n, false) || (bias && !valid_params(b, n, false))) return SVGD_ERR_INVALID_ARG;
    if (rows == 0) return SVGD_OK;
    if (!valid_input(x, dtype, rows) || !valid_output(y, dtype, n, rows, width) || !aligned_to(mean, 4) || !aligned_to(rstd, 4)) return SVGD_ERR_INVALID_ARG;
    const size_t stats = (size_t)n * rows * 4;
    const Extent written[3] = {extent(y, dtype, n, rows, width), extent(mean, mean ? stats : 0), extent(rstd, rstd ? stats : 0)};
    const Extent read[3] = {extent(x, dtype, n, rows, width), extent(weight, weight_stride, n, width),
                            bias ? extent(bias, bias_stride, n, width) : Extent{0, 0}};
    for (int a = 0; a < 3; ++a) {
        for (const Extent &r : read)
            if (written[a].meets(r)) return SVGD_ERR_INVALID_ARG;
        for (int o = 0; o < a; ++o)
            if (written[a].meets(written[o])) return SVGD_ERR_INVALID_ARG;
    }
    const NormShape s = forward_split(n, rows, width);
    return for_type(dtype, [&](auto t) {
        return for_team(width, [&](auto l, auto e) {
            using T = decltype(t);
            constexpr int L = decltype(l)::value, E = decltype(e)::value;
            norm_forward_kernel<T, L, E><<<n * s.blocks, kTeamBlock<L>, 0, (hipStream_t)stream>>>(s, in<T>(x), w, b, (float)eps, out<T>(y), mean, rstd);
            return launched();
        });
    });
}

size_t svgd_layer_norm_scratch(int n, int64_t rows, int64_t width)
{
    if (check_sizes(SVGD_F32, n, rows, width, SVGD_LAYER_MAX_NORM)) return 0;
    return (size_t)n * backward_split(n, rows, width).blocks * 2 * (size_t)width * 4;
}

int svgd_layer_norm_backward(int dtype, int n, int64_t rows, int64_t width, svgd_rows dy, svgd_rows x, const float *weight, int64_t weight_stride,
                             const float *mean, const float *rstd, svgd_rows dx, float *dweight, int64_t dweight_stride, float *dbias,
                             int64_t dbias_stride, int accumulate, void *scratch, size_t scratch_bytes, void *stream)
{
    if (const int rc = check_sizes(dtype, n, rows, width, SVGD_LAYER_MAX_NORM)) return rc;
    const Params w{weight, weight_stride, width}, dw{dweight, dweight_stride, width}, db{dbias, dbias_stride, width};
    if (!valid_params(w, n, false)) return SVGD_ERR_INVALID_ARG;
    for (const Params *g : {&dw, &db})
        if (g->p && (!valid_params(*g, n, true) || params_meet(*g, w, n))) return SVGD_ERR_INVALID_ARG;
    if (dw.p && db.p && params_meet(dw, db, n)) return SVGD_ERR_INVALID_ARG;
    const NormShape s = backward_split(n, rows, width);
    const bool params = dw.p || db.p;
    if (rows > 0) {
        const size_t need = params ? svgd_layer_norm_scratch(n, rows, width) : 0, stats = (size_t)n * rows * 4;
        if (!valid_input(dy, dtype, rows) || !valid_input(x, dtype, rows) || !mean || !rstd || !aligned_to(mean, 4) || !aligned_to(rstd, 4) ||
            (dx.data && !valid_output(dx, dtype, n, rows, width)) || (params && (!scratch || !aligned_to(scratch, 16) || scratch_bytes < need)))
            return SVGD_ERR_INVALID_ARG;
        const Extent read[5] = {extent(dy, dtype, n, rows, width), extent(x, dtype, n, rows, width), extent(mean, stats), extent(rstd, stats),
                                extent(weight, weight_stride, n, width)};
        const Extent written[4] = {dx.data ? extent(dx, dtype, n, rows, width) : Extent{0, 0}, extent(scratch, need),
                                   dw.p ? extent(dw.p, dw.stride, n, width) : Extent{0, 0}, db.p ? extent(db.p, db.stride, n, width) : Extent{0, 0}};
        for (int a = 0; a < 4; ++a) {
            for (int r = 0; r < (a < 2 ? 5 : 4); ++r) // (the gradients may lie between the weights, in the same rows: looked at above)
                if (written[a].meets(read[r])) return SVGD_ERR_INVALID_ARG;
            for (int o = 0; o < a && o < 2; ++o)
                if (written[a].meets(written[o])) return SVGD_ERR_INVALID_ARG;
        }
        if (dx.data || params) {
            const int rc = for_type(dtype, [&](auto t) {
                return for_team(width, [&](auto l, auto e) {
                    using T = decltype(t);
                    constexpr int L = decltype(l)::value, E = decltype(e)::value;
                    norm_backward_kernel<T, L, E><<<n * s.blocks, kTeamBlock<L>, 0, (hipStream_t)stream>>>(
                        s, in<T>(dy), in<T>(x), w, mean, rstd, out<T>(dx), params ? (float *)scratch : nullptr);
                    return launched();
                });
            });
            if (rc) return rc;
        }
    }
    if (!params || (rows == 0 && accumulate)) return SVGD_OK;
    const int groups = (int)((2 * width + 63) / 64);
    norm_reduce_kernel<<<n * groups, 64 * kReduceWaves, 0, (hipStream_t)stream>>>((const float *)scratch, rows > 0 ? s.blocks : 0, (int)width, groups, dw, db,
                                                                    accumulate != 0);
    return launched();
}

int svgd_dropout(int dtype, int n, int64_t rows, int64_t width, svgd_rows x, svgd_rows residual, svgd_rows y, double p, uint64_t seed, uint64_t call,
                 const int64_t *counter, void *stream)
{
    if (const int rc = check_sizes(dtype, n, rows, width, SVGD_MAX_D)) return rc;
    if (!(p >= 0.0 && p <= 1.0) || !aligned_to(counter, 8)) return SVGD_ERR_INVALID_ARG;
    if (rows == 0) return SVGD_OK;
    if (!valid_input(x, dtype, rows) || !valid_output(y, dtype, n, rows, width) || (residual.data && !valid_input(residual, dtype, rows))) return SVGD_ERR_INVALID_ARG;
    const Extent ye = extent(y, dtype, n, rows, width);
    for (const svgd_rows *r : {&x, &residual})
        if (r->data && ye.meets(extent(*r, dtype, n, rows, width)) && !same_rows(*r, y, n, rows)) return SVGD_ERR_INVALID_ARG;
    if (counter && ye.meets(extent(counter, 8))) return SVGD_ERR_INVALID_ARG;
    const double limit = std::nearbyint(p * 4294967296.0);
    DropArgs a{};
    const bool one_line = flat(x, n, rows, width) && flat(y, n, rows, width) && (!residual.data || flat(residual, n, rows, width));
    const int vec = 16 / (int)dtype_size(dtype);
    a.lines = one_line ? 1 : n * rows;
    a.per_particle = rows;
    a.width = one_line ? n * rows * width : width;
    a.packs = (a.width + vec - 1) / vec;
    a.base = splitmix64(splitmix64(seed) + call);
    a.counter = counter;
    a.none = limit >= 4294967296.0;
    a.limit = a.none ? 0xFFFFFFFFu : (uint32_t)limit;
    a.scale = a.none || p == 1.0 ? 0.f : (float)(1.0 / (1.0 - p));
    const int64_t groups = (a.lines * a.packs + 255) / 256;
    const int blocks = groups < 256 * 16 ? (int)groups : 256 * 16;
    return for_type(dtype, [&](auto t) {
        using T = decltype(t);
        const DropRows<const T> xr{(const T *)x.data, x.particle_stride, x.row_stride}, rr{(const T *)residual.data, residual.particle_stride, residual.row_stride};
        const DropRows<T> yr{(T *)y.data, y.particle_stride, y.row_stride};
        const hipStream_t st = (hipStream_t)stream;
        if (one_line && residual.data) dropout_kernel<T, true, true><<<blocks, 256, 0, st>>>(a, xr, rr, yr);
        else if (one_line) dropout_kernel<T, true, false><<<blocks, 256, 0, st>>>(a, xr, rr, yr);
        else if (residual.data) dropout_kernel<T, false, true><<<blocks, 256, 0, st>>>(a, xr, rr, yr);
        else dropout_kernel<T, false, false><<<blocks, 256, 0, st>>>(a, xr, rr, yr);
        return launched();
    });
}

} // extern "C"
