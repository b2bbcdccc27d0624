// Dropout from the counter-based generator of workloads.py (splitmix64: Steele, Lea & Flood, "Fast splittable pseudorandom
// number generators", OOPSLA 2014): a value's 32 random bits are a function of its index, so the backward pass makes them
// again and no mask is stored.  Two values share a 64-bit hash, whose two multiplications are what the pass computes; it is
// bound by memory.
#pragma once
#include "layer_common.hpp"

namespace svgd {

__host__ __device__ inline uint64_t splitmix64(uint64_t v)
{
    v += 0x9E3779B97F4A7C15ull;
    v = (v ^ (v >> 30)) * 0xBF58476D1CE4E5B9ull;
    v = (v ^ (v >> 27)) * 0x94D049BB133111EBull;
    return v ^ (v >> 31);
}

template <class T> struct DropRows {
    T *p;
    int64_t particle, row;
};

struct DropArgs {
    int64_t lines, per_particle; // lines of `width` values, `per_particle` of them to a particle
    int64_t width;
    int64_t packs;               // per line
    uint64_t base;
    const int64_t *counter;
    uint32_t limit;              // kept if not below
    bool none;                   // nothing is kept
    float scale;
};

// FLAT: one line.
template <class T, bool FLAT, bool RESIDUAL>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs a, DropRows<const T> x, DropRows<const T> residual, DropRows<T> y)
{
    constexpr int VEC = 16 / sizeof(T);
    const uint64_t base = a.counter ? splitmix64(a.base + (uint64_t)*a.counter) : a.base;
    const int64_t stride = (int64_t)gridDim.x * 256;
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < (FLAT ? a.packs : a.lines * a.packs); k += stride) {
        int64_t line = 0, col = k * VEC, xo = col, ro = col, yo = col;
        if constexpr (!FLAT) {
            line = k / a.packs;
            col = (k - line * a.packs) * VEC;
            const int64_t i = line / a.per_particle, t = line - i * a.per_particle;
            xo = i * x.particle + t * x.row + col;
            ro = i * residual.particle + t * residual.row + col;
            yo = i * y.particle + t * y.row + col;
        }
        const int left = a.width - col < VEC ? (int)(a.width - col) : VEC;
        const int64_t e0 = line * a.width + col;
        const bool odd = !FLAT && (e0 & 1);
        uint64_t h[VEC / 2 + 1];
#pragma unroll
        for (int q = 0; q < VEC / 2; ++q) h[q] = splitmix64(base + (uint64_t)(e0 >> 1) + q);
        h[VEC / 2] = odd ? splitmix64(base + (uint64_t)(e0 >> 1) + VEC / 2) : 0;
        float v[VEC], r[VEC];
        load_pack<T, VEC>(x.p + xo, left, v);
        if constexpr (RESIDUAL) load_pack<T, VEC>(residual.p + ro, left, r);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const uint32_t even_bits = e & 1 ? (uint32_t)h[e / 2] : (uint32_t)(h[e / 2] >> 32);
            const uint32_t odd_bits = e & 1 ? (uint32_t)(h[e / 2 + 1] >> 32) : (uint32_t)h[e / 2];
            const bool keep = (odd ? odd_bits : even_bits) >= a.limit && !a.none;
            v[e] = keep ? v[e] * a.scale : 0.f;
            if constexpr (RESIDUAL) v[e] += r[e];
        }
        store_pack<T, VEC>(y.p + yo, left, v);
    }
}

} // namespace svgd
