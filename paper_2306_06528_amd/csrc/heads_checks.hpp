// Checks of tensors with heads (include/svgd_attention.h).
#pragma once
#include "heads_rules.hpp"
#include "layer_common.hpp"

namespace svgd {

inline Extent extent(const svgd_heads &h, int dtype, const HeadSizes &s)
{
    if (!h.data || s.none()) return {0, 0};
    const uintptr_t last = (uintptr_t)(s.n - 1) * (uintptr_t)h.particle_stride + (uintptr_t)(s.batch - 1) * (uintptr_t)h.batch_stride +
                           (uintptr_t)(s.tokens - 1) * (uintptr_t)h.token_stride + (uintptr_t)(s.heads - 1) * (uintptr_t)h.head_stride + (uintptr_t)s.dim;
    return {(uintptr_t)h.data, (uintptr_t)h.data + last * dtype_size(dtype)};
}

inline bool valid_heads(const svgd_heads &h, int dtype, const HeadSizes &s)
{
    if (s.none()) return true; // (nothing is read or written)
    if (!h.data || !aligned_to(h.data, dtype_size(dtype))) return false;
    const int64_t strides[4] = {h.particle_stride, h.batch_stride, h.token_stride, h.head_stride}, sizes[4] = {s.n, s.batch, s.tokens, s.heads};
    for (int i = 0; i < 4; ++i)
        if (strides[i] < 0 || (sizes[i] > 1 && strides[i] > kMaxStride / sizes[i])) return false;
    return true;
}

// An output's heads must not overlap: sorted by stride, each dimension lies outside the ones before it.
inline bool valid_heads_output(const svgd_heads &h, int dtype, const HeadSizes &s)
{
    if (!valid_heads(h, dtype, s)) return false;
    if (s.none()) return true;
    struct { int64_t stride, size; } d[4] = {{h.particle_stride, s.n}, {h.batch_stride, s.batch}, {h.token_stride, s.tokens}, {h.head_stride, s.heads}};
    std::sort(d, d + 4, [](const auto &a, const auto &b) { return a.stride < b.stride; });
    int64_t span = s.dim;
    for (const auto &x : d) {
        if (x.size == 1) continue;
        if (x.stride < span) return false;
        span += (x.size - 1) * x.stride;
    }
    return true;
}

// What a call reads or writes: a tensor with heads, or a stretch of memory.
struct Region {
    Extent all;
    const svgd_heads *heads = nullptr;
    HeadSizes sizes{};
    int dtype = 0;
    Region(const Extent &e) : all(e) {}
    Region(const svgd_heads &h, int type, const HeadSizes &s) : all(extent(h, type, s)), heads(&h), sizes(s), dtype(type) {}
    bool meets(const Region &o) const
    {
        return all.meets(o.all) && !(heads && o.heads && heads_apart(*heads, sizes, *o.heads, o.sizes, (int64_t)dtype_size(dtype)));
    }
};

} // namespace svgd
