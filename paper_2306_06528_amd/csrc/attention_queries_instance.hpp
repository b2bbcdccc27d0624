// delta, and the kernels of one type that have queries of their own, and their launches.
#include "attention_backward.hpp"
#include "attention_launch.hpp"

template <> int svgd::attention_queries<SVGD_ATTENTION_TYPE>(AttnCall &c)
{
    typedef SVGD_ATTENTION_TYPE T;
    AttnArgs &a = c.a;
    const int64_t lines = (int64_t)a.n * a.batch * a.heads * a.t;
    attention_delta_kernel<T><<<(unsigned)ceil_div(lines, 16), 256, 0, c.stream>>>(a, in<T>(c.o), in<T>(c.d_o), const_cast<float *>(c.delta));
    if (const int rc = launched_ok()) return rc;
    if (!c.dq.data && !c.slope_rows) return SVGD_OK;
    const int blocks = row_blocks(a);
    set_grid(a, a.rows, 64 * blocks, 1);
    return with_dim(a.dim, [&](auto kd) {
        return with_two(blocks, [&](auto qb) {
            return with_truth(modified_scores(a), [&](auto mod) {
                attention_queries_kernel<T, decltype(kd)::value, decltype(qb)::value, decltype(mod)::value>
                    <<<a.per_die * 8, kAttnBlock, 0, c.stream>>>(a, in<T>(c.q), in<T>(c.k), in<T>(c.v), in<T>(c.d_o), c.lse, c.delta, out<T>(c.dq), c.slope_rows);
                return launched_ok();
            });
        });
    });
}
