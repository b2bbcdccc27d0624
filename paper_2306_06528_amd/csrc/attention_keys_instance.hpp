// The kernels of one type that have keys of their own, and their launches.
#include "attention_backward.hpp"
#include "attention_launch.hpp"

template <> int svgd::attention_keys<SVGD_ATTENTION_TYPE>(AttnCall &c)
{
    typedef SVGD_ATTENTION_TYPE T;
    AttnArgs &a = c.a;
    const int blocks = key_blocks(a);
    set_grid(a, a.s, 64 * blocks, 1);
    return with_dim(a.dim, [&](auto kd) {
        return with_two(blocks, [&](auto kb) {
            return with_truth(modified_scores(a), [&](auto mod) {
                attention_keys_kernel<T, decltype(kd)::value, decltype(kb)::value, decltype(mod)::value>
                    <<<a.per_die * 8, kAttnBlock, 0, c.stream>>>(a, in<T>(c.q), in<T>(c.k), in<T>(c.v), in<T>(c.d_o), c.lse, c.delta, out<T>(c.dk), out<T>(c.dv));
                return launched_ok();
            });
        });
    });
}
