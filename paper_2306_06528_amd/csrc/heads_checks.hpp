// Checks of tensors with heads (include/svgd_attention.h).
#pragma once
#include "layer_common.hpp"
#include "../../include/svgd_attention.h"

#include <algorithm>

namespace svgd {

struct HeadSizes {
    int64_t n, batch, tokens, heads, dim;
    bool none() const { return batch == 0 || tokens == 0 || heads == 0; }
};

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

// Whether two tensors of the same sizes lie side by side in the same rows, as views into the results of one linear map do: then their extents meet, they do not.
// (Same strides, and the second one's heads and values within the gap that the first one's leave in every token.)
inline bool side_by_side(const svgd_heads &a, int64_t a_heads, const svgd_heads &b, int64_t b_heads, int dtype, const HeadSizes &s)
{
    if (a.particle_stride != b.particle_stride || a.batch_stride != b.batch_stride || a.token_stride != b.token_stride || !a.data || !b.data) return false;
    const int64_t size = (int64_t)dtype_size(dtype), apart = ((intptr_t)b.data - (intptr_t)a.data);
    if (apart % size) return false;
    const int64_t d = apart / size, a_end = (a_heads - 1) * a.head_stride + s.dim, b_end = (b_heads - 1) * b.head_stride + s.dim;
    const int64_t lo = d < 0 ? -d : d, first_end = d < 0 ? b_end : a_end, second_end = d < 0 ? a_end : b_end; // the one that comes first begins at 0
    int64_t least = INT64_MAX;
    if (s.n > 1) least = std::min(least, a.particle_stride);
    if (s.batch > 1) least = std::min(least, a.batch_stride);
    if (s.tokens > 1) least = std::min(least, a.token_stride);
    return lo >= first_end && lo + second_end <= least;
}

} // namespace svgd
