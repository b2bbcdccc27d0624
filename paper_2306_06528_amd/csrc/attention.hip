// Host side of attention (include/svgd_attention.h): checks, scratch memory, the order of launches.
#include "attention_backward.hpp"
#include "attention_launch.hpp"
#include "heads_checks.hpp"

#include <cmath>

using namespace svgd;

namespace {

HeadSizes query_sizes(const svgd_attention &a) { return {a.n, a.batch, a.length, a.heads, a.dim}; }
HeadSizes key_sizes(const svgd_attention &a) { return {a.n, a.batch, a.keys, a.kv_heads, a.dim}; }

int check_sizes_of(const svgd_attention *a)
{
    if (!a || a->n < 1 || a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads || a->dim < 1 || a->batch < 0 || a->length < 0 || a->keys < 0)
        return SVGD_ERR_INVALID_ARG;
    if (a->n > SVGD_MAX_PARTICLES || a->dim > SVGD_ATTENTION_MAX_DIM || a->batch > SVGD_ATTENTION_MAX_BATCH || a->length > SVGD_ATTENTION_MAX_LENGTH ||
        a->keys > SVGD_ATTENTION_MAX_LENGTH || a->heads > SVGD_ATTENTION_MAX_HEADS)
        return SVGD_ERR_TOO_LARGE;
    const int64_t group = a->heads / a->kv_heads, rows = a->length * group, most = rows > a->keys ? rows : a->keys;
    if (group > SVGD_ATTENTION_MAX_GROUP || rows > SVGD_ATTENTION_MAX_LENGTH || a->n * a->batch * a->kv_heads > kMaxBlocks / (most < 64 ? 1 : ceil_div(most, 64)) ||
        a->n * a->batch * a->heads * (a->length < 1 ? 1 : a->length) > ((int64_t)1 << 28) - 16)
        return SVGD_ERR_TOO_LARGE;
    return SVGD_OK;
}

AttnArgs args_of(const svgd_attention &a)
{
    AttnArgs x{};
    x.n = a.n;
    x.batch = (int)a.batch;
    x.heads = a.heads;
    x.kv = a.kv_heads;
    x.group = a.heads / a.kv_heads;
    x.dim = a.dim;
    x.t = (int)a.length;
    x.s = (int)a.keys;
    x.rows = x.t * x.group;
    x.group_mul = x.group == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + x.group - 1) / x.group);
    x.causal = a.causal != 0;
    x.scale = (float)a.scale;
    x.cap = (float)a.cap;
    x.slopes = a.slopes;
    x.slopes_stride = a.slopes_stride;
    x.starts = a.starts;
    x.lengths = a.lengths;
    x.documents = a.documents;
    x.prefix = a.prefix;
    return x;
}

bool nothing(const svgd_attention &a) { return a.batch == 0 || (a.length == 0 && a.keys == 0); }
size_t lines_of(const svgd_attention &a) { return (size_t)a.n * a.batch * a.heads * a.length; }

// What both passes read besides the activations, as extents.
struct MaskExtents {
    Extent e[5];
    explicit MaskExtents(const svgd_attention &a)
    {
        const size_t each = (size_t)a.batch * 4;
        e[0] = extent(a.starts, a.starts ? each : 0);
        e[1] = extent(a.lengths, a.lengths ? each : 0);
        e[2] = extent(a.prefix, a.prefix ? each : 0);
        e[3] = extent(a.documents, a.documents ? each * a.keys : 0);
        e[4] = a.slopes ? extent(a.slopes, a.slopes_stride, a.n, a.heads) : Extent{0, 0};
    }
    bool meet(const Extent &x) const
    {
        for (const Extent &o : e)
            if (o.meets(x)) return true;
        return false;
    }
};

// Tokens, or the heads that share keys, further apart than the kernels' offsets within a tile reach.
bool far(const svgd_heads &h, int64_t together, int64_t tokens)
{
    return (tokens > 1 && h.token_stride >= kMaxTokenStride) || (together > 1 && h.head_stride >= kMaxTokenStride / together);
}

int check(int dtype, const svgd_attention *a, const svgd_heads &q, const svgd_heads &k, const svgd_heads &v)
{
    if (dtype < SVGD_F32 || dtype > SVGD_F16) return SVGD_ERR_INVALID_ARG;
    if (const int rc = check_sizes_of(a)) return rc;
    const float scale = (float)a->scale, cap = (float)a->cap; // (what does not fit fp32 is refused)
    if (!std::isfinite(scale) || !(scale > 0.f) || !std::isfinite(cap) || !(a->cap >= 0.0) || (a->cap > 0.0 && cap < 1e-30f) || scale < 1e-30f) return SVGD_ERR_INVALID_ARG;
    // what the kernels make of them (Modified): times log2 e, and their quotient, which as a subnormal would have few digits
    if (!std::isfinite(scale * kLog2e) || !std::isfinite(cap * kLog2e) || (cap > 0.f && !std::isnormal(scale / cap))) return SVGD_ERR_INVALID_ARG;
    if (a->slopes && !valid_params({a->slopes, a->slopes_stride, a->heads}, a->n, false)) return SVGD_ERR_INVALID_ARG;
    if (!aligned_to(a->starts, 4) || !aligned_to(a->lengths, 4) || !aligned_to(a->documents, 4) || !aligned_to(a->prefix, 4)) return SVGD_ERR_INVALID_ARG;
    if (far(q, a->heads / a->kv_heads, a->length) || far(k, 1, a->keys) || far(v, 1, a->keys)) return SVGD_ERR_TOO_LARGE;
    if (!valid_heads(q, dtype, query_sizes(*a)) || !valid_heads(k, dtype, key_sizes(*a)) || !valid_heads(v, dtype, key_sizes(*a))) return SVGD_ERR_INVALID_ARG;
    return SVGD_OK;
}

template <class F> int for_type(int dtype, F f) { return dtype == SVGD_F32 ? f(float{}) : dtype == SVGD_BF16 ? f(bf16_t{}) : f(f16_t{}); }


size_t rounded(size_t floats) { return (floats + 3) / 4 * 4; }

// Scratch memory of the backward pass, in floats: delta, the slopes' rows, where queries' rows are in parts these parts' sums of dz (and
// with slopes two more), parts' sums of dq (and of the keys' means, which 16 bits need) or of dk and dv, which come after them.
struct BackwardScratch {
    size_t slopes, sums, partial, total;
    explicit BackwardScratch(const svgd_attention &p)
    {
        const AttnArgs a = args_of(p);
        const size_t lines = lines_of(p), key_lines = (size_t)p.n * p.batch * p.kv_heads * p.keys;
        const size_t qs = query_splits(a), ks = key_splits(a), ld = padded_dim(a);
        slopes = rounded(lines);
        sums = slopes + (p.slopes ? rounded(lines) : 0);
        partial = sums + (qs > 1 ? rounded(lines * qs * (p.slopes ? 3 : 1)) : 0);
        const size_t of_q = qs > 1 ? qs * lines * 2 * ld : 0, of_k = ks > 1 ? ks * key_lines * 2 * ld : 0;
        total = partial + (of_q > of_k ? of_q : of_k);
    }
};

} // namespace

extern "C" {

size_t svgd_attention_forward_scratch(const svgd_attention *p)
{
    if (check_sizes_of(p) || nothing(*p) || p->length == 0) return 0;
    const AttnArgs a = args_of(*p);
    const int splits = forward_splits(a);
    return splits == 1 ? 0 : splits * lines_of(*p) * (padded_dim(a) + 1) * 4;
}

int svgd_attention_forward(int dtype, const svgd_attention *p, svgd_heads q, svgd_heads k, svgd_heads v, svgd_heads o, float *lse, void *scratch, size_t scratch_bytes,
                           void *stream)
{
    if (const int rc = check(dtype, p, q, k, v)) return rc;
    if (p->batch == 0 || p->length == 0) return SVGD_OK;
    const size_t need = svgd_attention_forward_scratch(p), stats = lines_of(*p) * 4;
    if (!valid_heads_output(o, dtype, query_sizes(*p)) || !aligned_to(lse, 4) || (need && (!scratch || !aligned_to(scratch, 16) || scratch_bytes < need))) return SVGD_ERR_INVALID_ARG;
    const HeadSizes qs = query_sizes(*p), ks = key_sizes(*p);
    const Region written[3] = {{o, dtype, qs}, extent(lse, lse ? stats : 0), extent(scratch, need)}, read[3] = {{q, dtype, qs}, {k, dtype, ks}, {v, dtype, ks}};
    const MaskExtents masks(*p);
    for (int i = 0; i < 3; ++i) {
        for (const Region &r : read)
            if (written[i].meets(r)) return SVGD_ERR_INVALID_ARG;
        if (masks.meet(written[i].all)) return SVGD_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (written[i].meets(written[j])) return SVGD_ERR_INVALID_ARG;
    }
    AttnCall c{};
    c.a = args_of(*p);
    c.q = q;
    c.k = k;
    c.v = v;
    c.o = o;
    c.lse_out = lse;
    c.partial = (float *)scratch;
    c.partial_lse = c.partial ? c.partial + (size_t)forward_splits(c.a) * lines_of(*p) * padded_dim(c.a) : nullptr;
    c.stream = (hipStream_t)stream;
    return for_type(dtype, [&](auto t) { return attention_forward<decltype(t)>(c); });
}

size_t svgd_attention_scratch(const svgd_attention *p)
{
    if (check_sizes_of(p)) return 0;
    return BackwardScratch(*p).total * 4;
}

int svgd_attention_backward(int dtype, const svgd_attention *p, svgd_heads d_o, svgd_heads q, svgd_heads k, svgd_heads v, svgd_heads o, const float *lse, svgd_heads dq, svgd_heads dk,
                            svgd_heads dv, float *dslopes, int64_t dslopes_stride, int accumulate, void *scratch, size_t scratch_bytes, void *stream)
{
    if (const int rc = check(dtype, p, q, k, v)) return rc;
    const HeadSizes qs = query_sizes(*p), ks = key_sizes(*p);
    if (far(d_o, p->heads / p->kv_heads, p->length)) return SVGD_ERR_TOO_LARGE;
    const size_t need = svgd_attention_scratch(p), stats = lines_of(*p) * 4;
    const Params slopes{p->slopes, p->slopes_stride, p->heads}, grads{dslopes, dslopes_stride, p->heads};
    if (dslopes && (!p->slopes || !valid_params(grads, p->n, true) || params_meet(grads, slopes, p->n))) return SVGD_ERR_INVALID_ARG;
    if (!valid_heads(d_o, dtype, qs) || !valid_heads(o, dtype, qs) || (stats && (!lse || !aligned_to(lse, 4))) || (dq.data && !valid_heads_output(dq, dtype, qs)) ||
        (dk.data && !valid_heads_output(dk, dtype, ks)) || (dv.data && !valid_heads_output(dv, dtype, ks)) ||
        (need && (!scratch || !aligned_to(scratch, 16) || scratch_bytes < need)))
        return SVGD_ERR_INVALID_ARG;
    const Region written[5] = {{dq, dtype, qs}, {dk, dtype, ks}, {dv, dtype, ks}, extent(scratch, need), dslopes ? extent(dslopes, dslopes_stride, p->n, p->heads) : Extent{0, 0}};
    const Region read[6] = {{q, dtype, qs}, {k, dtype, ks}, {v, dtype, ks}, {d_o, dtype, qs}, {o, dtype, qs}, extent(lse, stats)};
    const MaskExtents masks(*p);
    for (int i = 0; i < 5; ++i) {
        for (const Region &r : read)
            if (written[i].meets(r)) return SVGD_ERR_INVALID_ARG;
        for (int m = 0; m < (i < 4 ? 5 : 4); ++m) // (the slopes' gradients may lie between the slopes, in the same rows: looked at above)
            if (masks.e[m].meets(written[i].all)) return SVGD_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (written[i].meets(written[j])) return SVGD_ERR_INVALID_ARG;
    }
    AttnCall c{};
    c.a = args_of(*p);
    c.q = q;
    c.k = k;
    c.v = v;
    c.o = o;
    c.d_o = d_o;
    c.dq = dq;
    c.dk = dk;
    c.dv = dv;
    c.lse = lse;
    c.delta = (const float *)scratch;
    const BackwardScratch parts(*p);
    c.slope_rows = dslopes ? (float *)scratch + parts.slopes : nullptr;
    c.row_sums = (float *)scratch + parts.sums;
    c.partial = (float *)scratch + parts.partial;
    c.stream = (hipStream_t)stream;
    if (p->batch > 0 && p->length > 0) {
        const int rc = for_type(dtype, [&](auto t) { return attention_queries<decltype(t)>(c); });
        if (rc) return rc;
    }
    if (p->batch > 0 && p->keys > 0 && (dk.data || dv.data)) {
        const int rc = for_type(dtype, [&](auto t) { return attention_keys<decltype(t)>(c); });
        if (rc) return rc;
    }
    if (!dslopes || (accumulate && (p->batch == 0 || p->length == 0))) return SVGD_OK;
    attention_slopes_kernel<<<p->n * p->heads, 256, 0, c.stream>>>(c.a, c.slope_rows, dslopes, dslopes_stride, accumulate != 0);
    return launched_ok();
}

} // extern "C"
