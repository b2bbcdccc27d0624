// Host side of the norms of queries and keys with their rotation (include/svgd_attention.h): checks and launches.
#include "heads_checks.hpp"
#include "norm_kernels.hpp"
#include "rotary_kernels.hpp"

#include <cmath>

using namespace svgd;

namespace {

int launched() { return hipGetLastError() == hipSuccess ? SVGD_OK : SVGD_ERR_DEVICE; }
template <class F> int for_type(int dtype, F f) { return dtype == SVGD_F32 ? f(float{}) : dtype == SVGD_BF16 ? f(bf16_t{}) : f(f16_t{}); }
template <class T> Heads<const T> in(const svgd_heads &h) { return {(const T *)h.data, h.particle_stride, h.batch_stride, h.token_stride, h.head_stride}; }
template <class T> Heads<T> out(const svgd_heads &h) { return {(T *)h.data, h.particle_stride, h.batch_stride, h.token_stride, h.head_stride}; }

// Lanes for a head.
template <class T, class F> int for_team(int dim, F f)
{
    using std::integral_constant;
    const int pieces = (dim * (int)sizeof(T) + 15) / 16;
    if (pieces <= 4) return f(integral_constant<int, 4>{});
    if (pieces <= 8) return f(integral_constant<int, 8>{});
    if (pieces <= 16) return f(integral_constant<int, 16>{});
    if (pieces <= 32) return f(integral_constant<int, 32>{});
    return f(integral_constant<int, 64>{});
}

HeadSizes q_sizes(const svgd_rotary &p) { return {p.n, p.batch, p.length, p.heads, p.dim}; }
HeadSizes k_sizes(const svgd_rotary &p) { return {p.n, p.batch, p.length, p.kv_heads, p.dim}; }

int check_sizes_of(const svgd_rotary *p)
{
    if (!p || p->n < 1 || p->heads < 0 || p->kv_heads < 0 || p->dim < 1 || p->pairs < 0 || p->batch < 0 || p->length < 0) return SVGD_ERR_INVALID_ARG;
    if (p->n > SVGD_MAX_PARTICLES || p->dim > SVGD_ROTARY_MAX_DIM || p->batch > SVGD_ATTENTION_MAX_BATCH || p->length > SVGD_ATTENTION_MAX_LENGTH || p->heads > SVGD_ATTENTION_MAX_HEADS ||
        p->kv_heads > SVGD_ATTENTION_MAX_HEADS || (p->length > 0 && p->batch > ((int64_t)1 << 31) / p->length))
        return SVGD_ERR_TOO_LARGE;
    return 2 * p->pairs > p->dim ? SVGD_ERR_INVALID_ARG : SVGD_OK;
}

int check(int dtype, const svgd_rotary *p)
{
    if (dtype < SVGD_F32 || dtype > SVGD_F16) return SVGD_ERR_INVALID_ARG;
    if (const int rc = check_sizes_of(p)) return rc;
    if (!std::isfinite(p->eps) || p->eps < 0 || (p->q_weight == nullptr) != (p->k_weight == nullptr)) return SVGD_ERR_INVALID_ARG;
    if (p->q_weight && (!valid_params({p->q_weight, p->q_weight_stride, p->dim}, p->n, false) || !valid_params({p->k_weight, p->k_weight_stride, p->dim}, p->n, false))) return SVGD_ERR_INVALID_ARG;
    if (p->pairs > 0 && p->batch > 0 && p->length > 0 &&
        (!p->frequencies || !aligned_to(p->frequencies, 8) || !p->positions || !aligned_to(p->positions, 8) || p->positions_stride < 0 || p->positions_stride > kMaxStride / p->batch))
        return SVGD_ERR_INVALID_ARG;
    return SVGD_OK;
}

// Tokens of a particle to workgroups: enough of these for the part (with kTokens tokens each, or fewer where tokens are few).
RotaryArgs args_of(const svgd_rotary &p, int64_t most)
{
    RotaryArgs a{};
    a.dim = p.dim;
    a.pairs = p.pairs;
    a.interleaved = p.interleaved != 0;
    a.length = (int)p.length;
    a.tokens = p.batch * p.length;
    a.frequencies = p.frequencies;
    a.positions = p.positions;
    a.positions_stride = p.positions_stride;
    a.eps = (float)p.eps;
    const int64_t blocks = most / p.n > 1 ? most / p.n : 1;
    a.per = (a.tokens + blocks - 1) / blocks;
    if (a.per > kTokens) a.per = (a.per + kTokens - 1) / kTokens * kTokens;
    if (a.per < 1) a.per = 1;
    a.blocks = (int)((a.tokens + a.per - 1) / a.per);
    return a;
}
// (Forward, 8 x 8 x 197 x 12 heads of 64 bf16: 8,192 workgroups 30 us, 2,048 17, fewer angles being formed twice.  Backward, 8 x 2 x 4,096
// x 20 heads of 128 bf16: 768, as many as are there at a time, 233 us, 1,024 286, 2,048 243.)
constexpr int64_t kForwardBlocks = 2048, kBackwardBlocks = 768;

struct Reads { // besides the activations
    Extent e[4];
    explicit Reads(const svgd_rotary &p)
    {
        e[0] = extent(p.frequencies, p.pairs > 0 && p.frequencies ? (size_t)p.pairs * 8 : 0);
        e[1] = extent(p.positions, p.pairs > 0 && p.positions && p.batch > 0 ? ((size_t)(p.batch - 1) * p.positions_stride + p.length) * 8 : 0);
        e[2] = p.q_weight ? extent(p.q_weight, p.q_weight_stride, p.n, p.dim) : Extent{0, 0};
        e[3] = p.k_weight ? extent(p.k_weight, p.k_weight_stride, p.n, p.dim) : Extent{0, 0};
    }
};

} // namespace

extern "C" {

int svgd_qk_norm_rotary_forward(int dtype, const svgd_rotary *p, svgd_heads q, svgd_heads k, svgd_heads q_out, svgd_heads k_out, void *stream)
{
    if (const int rc = check(dtype, p)) return rc;
    const HeadSizes qs = q_sizes(*p), ks = k_sizes(*p);
    if (!valid_heads(q, dtype, qs) || !valid_heads(k, dtype, ks) || !valid_heads_output(q_out, dtype, qs) || !valid_heads_output(k_out, dtype, ks)) return SVGD_ERR_INVALID_ARG;
    if (qs.none() && ks.none()) return SVGD_OK;
    const Reads reads(*p);
    const Region written[2] = {{q_out, dtype, qs}, {k_out, dtype, ks}}, inputs[2] = {{q, dtype, qs}, {k, dtype, ks}};
    for (const Region &w : written) {
        for (const Extent &r : reads.e)
            if (w.meets(r)) return SVGD_ERR_INVALID_ARG;
        for (const Region &r : inputs)
            if (w.meets(r)) return SVGD_ERR_INVALID_ARG;
    }
    if (written[0].meets(written[1])) return SVGD_ERR_INVALID_ARG;
    const RotaryArgs a = args_of(*p, kForwardBlocks);
    return for_type(dtype, [&](auto t) {
        using T = decltype(t);
        return for_team<T>(p->dim, [&](auto l) {
            const RotaryKinds<T> kinds{{{in<T>(q), {}, out<T>(q_out), {p->q_weight, p->q_weight_stride, p->dim}, p->heads},
                                        {in<T>(k), {}, out<T>(k_out), {p->k_weight, p->k_weight_stride, p->dim}, p->kv_heads}}};
            constexpr int L = decltype(l)::value;
            if (p->dim * sizeof(T) % 16 == 0) rotary_forward_kernel<T, L, true><<<p->n * a.blocks, kRotaryBlock, 0, (hipStream_t)stream>>>(a, kinds);
            else rotary_forward_kernel<T, L, false><<<p->n * a.blocks, kRotaryBlock, 0, (hipStream_t)stream>>>(a, kinds);
            return launched();
        });
    });
}

size_t svgd_qk_norm_rotary_scratch(const svgd_rotary *p)
{
    if (check_sizes_of(p)) return 0;
    return (size_t)p->n * args_of(*p, kBackwardBlocks).blocks * 2 * p->dim * 4;
}

int svgd_qk_norm_rotary_backward(int dtype, const svgd_rotary *p, svgd_heads dq_out, svgd_heads dk_out, svgd_heads q, svgd_heads k, svgd_heads dq, svgd_heads dk, float *dq_weight,
                                 int64_t dq_weight_stride, float *dk_weight, int64_t dk_weight_stride, int accumulate, void *scratch, size_t scratch_bytes, void *stream)
{
    if (const int rc = check(dtype, p)) return rc;
    const HeadSizes qs = q_sizes(*p), ks = k_sizes(*p);
    const bool norm = p->q_weight != nullptr, params = dq_weight || dk_weight;
    const Params w[2] = {{p->q_weight, p->q_weight_stride, p->dim}, {p->k_weight, p->k_weight_stride, p->dim}};
    const Params g[2] = {{dq_weight, dq_weight_stride, p->dim}, {dk_weight, dk_weight_stride, p->dim}};
    if (params && !norm) return SVGD_ERR_INVALID_ARG;
    for (const Params &x : g)
        if (x.p && (!valid_params(x, p->n, true) || params_meet(x, w[0], p->n) || params_meet(x, w[1], p->n))) return SVGD_ERR_INVALID_ARG;
    if (g[0].p && g[1].p && params_meet(g[0], g[1], p->n)) return SVGD_ERR_INVALID_ARG;
    if (!valid_heads(dq_out, dtype, qs) || !valid_heads(dk_out, dtype, ks) || (norm && (!valid_heads(q, dtype, qs) || !valid_heads(k, dtype, ks))) ||
        (dq.data && !valid_heads_output(dq, dtype, qs)) || (dk.data && !valid_heads_output(dk, dtype, ks)))
        return SVGD_ERR_INVALID_ARG;
    const size_t need = params ? svgd_qk_norm_rotary_scratch(p) : 0;
    if (need && (!scratch || !aligned_to(scratch, 16) || scratch_bytes < need)) return SVGD_ERR_INVALID_ARG;
    const bool none = qs.none() && ks.none();
    if (!none) {
        const Reads reads(*p);
        const Extent work = extent(scratch, need);
        const Region written[2] = {{dq, dtype, qs}, {dk, dtype, ks}};
        Extent grads[2];
        for (int i = 0; i < 2; ++i) grads[i] = g[i].p ? extent(g[i].p, g[i].stride, p->n, p->dim) : Extent{0, 0};
        const svgd_heads *const acts[4] = {&dq_out, &dk_out, &q, &k};
        for (int i = 0; i < (norm ? 4 : 2); ++i) {
            const HeadSizes &s = i % 2 ? ks : qs;
            const Region e(*acts[i], dtype, s);
            if (work.meets(e.all) || grads[0].meets(e.all) || grads[1].meets(e.all)) return SVGD_ERR_INVALID_ARG;
            if (written[0].meets(e) || written[1].meets(e)) return SVGD_ERR_INVALID_ARG;
        }
        if (written[0].meets(written[1])) return SVGD_ERR_INVALID_ARG;
        for (const Region &x : written) {
            if (work.meets(x.all) || grads[0].meets(x.all) || grads[1].meets(x.all)) return SVGD_ERR_INVALID_ARG;
            for (const Extent &r : reads.e)
                if (x.meets(r)) return SVGD_ERR_INVALID_ARG;
        }
        for (const Extent &r : reads.e)
            if (work.meets(r)) return SVGD_ERR_INVALID_ARG;
        for (const Extent &x : grads)
            if (work.meets(x) || x.meets(reads.e[0]) || x.meets(reads.e[1])) return SVGD_ERR_INVALID_ARG;
    }
    const RotaryArgs a = args_of(*p, kBackwardBlocks);
    if (!none && (dq.data || dk.data || params)) {
        const int rc = for_type(dtype, [&](auto t) {
            using T = decltype(t);
            return for_team<T>(p->dim, [&](auto l) {
                const RotaryKinds<T> kinds{{{in<T>(q), in<T>(dq_out), out<T>(dq), w[0], p->heads}, {in<T>(k), in<T>(dk_out), out<T>(dk), w[1], p->kv_heads}}};
                constexpr int L = decltype(l)::value;
                float *const partial = params ? (float *)scratch : nullptr;
                if (p->dim * sizeof(T) % 16 == 0) rotary_backward_kernel<T, L, true><<<p->n * a.blocks, kRotaryBlock, 0, (hipStream_t)stream>>>(a, kinds, partial);
                else rotary_backward_kernel<T, L, false><<<p->n * a.blocks, kRotaryBlock, 0, (hipStream_t)stream>>>(a, kinds, partial);
                return launched();
            });
        });
        if (rc) return rc;
    }
    if (!params || (none && accumulate)) return SVGD_OK;
    const int groups = (2 * p->dim + 63) / 64;
    norm_reduce_kernel<<<p->n * groups, 64 * kReduceWaves, 0, (hipStream_t)stream>>>((const float *)scratch, none ? 0 : a.blocks, p->dim, groups, g[0], g[1], accumulate != 0);
    return launched();
}

} // extern "C"
