// delta, and the kernels of one type that have queries of their own, and their launches.
#include "attention_backward.hpp"
#include "attention_launch.hpp"

template <> int svgd::attention_queries<SVGD_ATTENTION_TYPE>(AttnCall &c)
{
    typedef SVGD_ATTENTION_TYPE T;
    AttnArgs &a = c.a;
    const int64_t lines = (int64_t)a.n * a.batch * a.heads * a.t;
    float *const delta = const_cast<float *>(c.delta);
    if constexpr (!kRestore<T>)
        if (!c.dq.data && !c.slope_rows) {
            attention_delta_kernel<T><<<(unsigned)ceil_div(lines, 16), 256, 0, c.stream>>>(a, in<T>(c.o), in<T>(c.d_o), delta);
            return launched_ok();
        }
    int rc = with_dim(a.dim, [&](auto kd) {
        return with_truth(modified_scores(a), [&](auto mod) {
            constexpr int KD = decltype(kd)::value;
            constexpr bool MOD = decltype(mod)::value;
            set_grid(a, a.rows, 16 * kAttnWaves, query_splits(a));
            const int grid = a.per_die * 8;
            attention_queries_kernel<T, KD, MOD>
                <<<grid, kAttnBlock, 0, c.stream>>>(a, in<T>(c.q), in<T>(c.k), in<T>(c.v), in<T>(c.d_o), in<T>(c.o), c.lse, delta, out<T>(c.dq), c.slope_rows, c.row_sums,
                                                                            c.partial);
            return launched_ok();
        });
    });
    if (rc || a.splits == 1) return rc;
    if (c.dq.data || kRestore<T>) {
        const int ld = padded_dim(a);
        attention_query_sums_kernel<T><<<(unsigned)ceil_div(lines * (c.dq.data ? ld / 4 : 1), 256), 256, 0, c.stream>>>(a, ld, c.partial, c.row_sums, delta, out<T>(c.dq));
        if ((rc = launched_ok())) return rc;
    }
    if (c.slope_rows) {
        attention_slope_rows_kernel<<<(unsigned)ceil_div(lines, 256), 256, 0, c.stream>>>(a, c.row_sums, c.slope_rows);
        rc = launched_ok();
    }
    return rc;
}
