// The forward kernels of one type and their launches.
#include "attention_forward.hpp"
#include "attention_launch.hpp"

template <> int svgd::attention_forward<SVGD_ATTENTION_TYPE>(AttnCall &c)
{
    typedef SVGD_ATTENTION_TYPE T;
    AttnArgs &a = c.a;
    const int rc = with_dim(a.dim, [&](auto kd) {
        return with_truth(modified_scores(a), [&](auto mod) {
            constexpr int KD = decltype(kd)::value;
            constexpr bool MOD = decltype(mod)::value;
            if (few_rows(a)) {
                set_grid(a, a.rows, 16 * kAttnWaves, forward_splits(a));
                attention_few_kernel<T, KD, MOD><<<a.per_die * 8, kAttnBlock, 0, c.stream>>>(a, in<T>(c.q), in<T>(c.k), in<T>(c.v), out<T>(c.o), c.lse_out, c.partial, c.partial_lse);
                return launched_ok();
            }
            constexpr bool kTwo = two_forward(sizeof(T), KD, MOD);
            const bool two = kTwo && many_forward(a);
            set_grid(a, a.rows, 16 * kAttnWaves * (two ? 2 : 1), forward_splits(a));
            const int grid = a.per_die * 8;
            if constexpr (kTwo)
                if (two) {
                    attention_forward_kernel<T, KD, 2, MOD><<<grid, kAttnBlock, 0, c.stream>>>(a, in<T>(c.q), in<T>(c.k), in<T>(c.v), out<T>(c.o), c.lse_out, c.partial, c.partial_lse);
                    return launched_ok();
                }
            attention_forward_kernel<T, KD, 1, MOD><<<grid, kAttnBlock, 0, c.stream>>>(a, in<T>(c.q), in<T>(c.k), in<T>(c.v), out<T>(c.o), c.lse_out, c.partial, c.partial_lse);
            return launched_ok();
        });
    });
    if (rc || a.splits == 1) return rc;
    const int ld = padded_dim(a);
    const int64_t threads = (int64_t)a.n * a.batch * a.heads * a.t * (ld / 4);
    attention_join_kernel<T><<<(unsigned)ceil_div(threads, 256), 256, 0, c.stream>>>(a, ld, c.partial, c.partial_lse, out<T>(c.o), c.lse_out);
    return launched_ok();
}
