// Whether tensors with heads meet in memory: plain numbers, no HIP.
#pragma once
#include "../../include/svgd_attention.h"

#include <algorithm>
#include <cstdint>

namespace svgd {

struct HeadSizes {
    int64_t n, batch, tokens, heads, dim;
    bool none() const { return batch == 0 || tokens == 0 || heads == 0; }
};

// Whether no value of one is one of the other's (`size` bytes each), where their addresses go through each other: the queries', keys' and
// values' parts of one linear map's results, or of its gradient.  They lie apart if their outer dimensions are the same, if what is inside
// of these (the values, and mostly the heads) are two stretches side by side, and if from one step of an outer dimension to the next it is
// as far as both together and all that is nearer.  Every choice of outer dimensions is tried; strides are valid ones (valid_heads).
inline bool heads_apart(const svgd_heads &a, const HeadSizes &as, const svgd_heads &b, const HeadSizes &bs, int64_t size)
{
    if (!a.data || !b.data || as.none() || bs.none()) return true;
    struct Dimension { int64_t a_stride, a_size, b_stride, b_size; };
    const Dimension all[4] = {{a.particle_stride, as.n, b.particle_stride, bs.n}, {a.batch_stride, as.batch, b.batch_stride, bs.batch},
                              {a.token_stride, as.tokens, b.token_stride, bs.tokens}, {a.head_stride, as.heads, b.head_stride, bs.heads}};
    const int64_t from = (int64_t)((uintptr_t)b.data - (uintptr_t)a.data); // bytes
    for (int outer = 0; outer < 16; ++outer) {
        int64_t a_span = as.dim, b_span = bs.dim;
        Dimension out[4];
        int count = 0;
        bool same = true;
        for (int d = 0; d < 4; ++d) {
            const Dimension &x = all[d];
            if (outer >> d & 1) {
                same = same && x.a_size == x.b_size && (x.a_size == 1 || x.a_stride == x.b_stride);
                if (x.a_size > 1) out[count++] = x;
            } else {
                a_span += (x.a_size - 1) * x.a_stride;
                b_span += (x.b_size - 1) * x.b_stride;
            }
        }
        if (!same) continue;
        const int64_t a_bytes = a_span * size, b_bytes = b_span * size;
        if (from < a_bytes && -from < b_bytes) continue; // the stretches meet
        std::sort(out, out + count, [](const Dimension &x, const Dimension &y) { return x.a_stride < y.a_stride; });
        int64_t reach = std::max(a_bytes, from + b_bytes) - std::min<int64_t>(0, from);
        bool apart = true;
        for (int k = 0; k < count && apart; ++k) {
            apart = out[k].a_stride * size >= reach;
            reach += (out[k].a_size - 1) * out[k].a_stride * size;
        }
        if (apart) return true;
    }
    return false;
}

} // namespace svgd
