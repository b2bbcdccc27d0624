// What a call of attention launches, by sizes alone (attention_rules.hpp).  The kernels' instances are compiled type by type
// (attention_*_<type>.hip).
#pragma once
#include "attention_common.hpp"

namespace svgd {

struct AttnCall {
    AttnArgs a;
    svgd_heads q, k, v, o, d_o, dq, dk, dv;
    const float *lse, *delta;
    float *lse_out, *partial, *partial_lse, *slope_rows, *row_sums;
    hipStream_t stream;
};

template <class T> Heads<const T> in(const svgd_heads &h) { return {(const T *)h.data, h.particle_stride, h.batch_stride, h.token_stride, h.head_stride}; }
template <class T> Heads<T> out(const svgd_heads &h) { return {(T *)h.data, h.particle_stride, h.batch_stride, h.token_stride, h.head_stride}; }

// Tiles of `own` rows each of `size`, the streamed ones in `splits` parts; the workgroups' numbers.
inline void set_grid(AttnArgs &a, int64_t size, int own, int splits)
{
    a.tiles = (int)ceil_div(size, own);
    a.splits = splits;
    a.total = (int)((int64_t)a.n * a.batch * a.kv * a.tiles * splits);
    a.per_die = (a.total + 7) / 8;
}

inline int padded_dim(const AttnArgs &a) { return (a.dim + 31) / 32 * 32; }

template <class F> int with_dim(int dim, F f)
{
    using std::integral_constant;
    switch (dim_kind(dim)) {
    case 0: return f(integral_constant<int, 0>{});
    case 1: return f(integral_constant<int, 1>{});
    case 2: return f(integral_constant<int, 2>{});
    case 3: return f(integral_constant<int, 3>{});
    default: return f(integral_constant<int, 4>{});
    }
}
template <class F> int with_truth(bool b, F f) { return b ? f(std::true_type{}) : f(std::false_type{}); }

inline bool modified_scores(const AttnArgs &a) { return a.cap > 0.f || a.slopes; }
inline int launched_ok() { return hipGetLastError() == hipSuccess ? SVGD_OK : SVGD_ERR_DEVICE; }

template <class T> int attention_forward(AttnCall &c);
template <class T> int attention_queries(AttnCall &c);
template <class T> int attention_keys(AttnCall &c);

} // namespace svgd
