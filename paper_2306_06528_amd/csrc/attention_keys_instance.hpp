// The kernels of one type that have keys of their own, and their launches.
#include "attention_backward.hpp"
#include "attention_launch.hpp"

template <> int svgd::attention_keys<SVGD_ATTENTION_TYPE>(AttnCall &c)
{
    typedef SVGD_ATTENTION_TYPE T;
    AttnArgs &a = c.a;
    const int rc = with_dim(a.dim, [&](auto kd) {
        return with_truth(modified_scores(a), [&](auto mod) {
            constexpr int KD = decltype(kd)::value;
            constexpr bool MOD = decltype(mod)::value;
            constexpr bool kTwo = two_keys(sizeof(T), KD, MOD);
            const bool two = kTwo && many_keys(a);
            set_grid(a, a.s, 16 * kAttnWaves * (two ? 2 : 1), key_splits(a));
            const int grid = a.per_die * 8;
            if constexpr (kTwo)
                if (two) {
                    attention_keys_kernel<T, KD, 2, MOD>
                        <<<grid, kAttnBlock, 0, c.stream>>>(a, in<T>(c.q), in<T>(c.k), in<T>(c.v), in<T>(c.d_o), c.lse, c.delta, out<T>(c.dk), out<T>(c.dv), c.partial);
                    return launched_ok();
                }
            attention_keys_kernel<T, KD, 1, MOD>
                <<<grid, kAttnBlock, 0, c.stream>>>(a, in<T>(c.q), in<T>(c.k), in<T>(c.v), in<T>(c.d_o), c.lse, c.delta, out<T>(c.dk), out<T>(c.dv), c.partial);
            return launched_ok();
        });
    });
    if (rc || a.splits == 1) return rc;
    const int ld = padded_dim(a);
    const int64_t lines = (int64_t)a.n * a.batch * a.kv * a.s;
    attention_key_sums_kernel<T><<<(unsigned)ceil_div(lines * (ld / 2), 256), 256, 0, c.stream>>>(a, ld, c.partial, out<T>(c.dk), out<T>(c.dv));
    return launched_ok();
}
