// What the kernels of the particles' own layers share: activation types, 16-byte pieces of rows, checks of arguments.
#pragma once
#include "../../include/svgd_layers.h"
#include "common.hpp"

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

namespace svgd {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// VEC values of T that are as aligned as T is: rows may start anywhere.  (Global loads and stores of 16 bytes need no
// more than that here.)
template <class T, int VEC> struct Pack {
    typedef T raw __attribute__((ext_vector_type(VEC)));
    typedef raw type __attribute__((aligned(sizeof(T))));
};

template <class T, int VEC>
__device__ __forceinline__ void load_pack(const T *__restrict__ p, int left, float (&v)[VEC])
{
    if (left >= VEC) {
        const typename Pack<T, VEC>::raw r = *reinterpret_cast<const typename Pack<T, VEC>::type *>(p);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = (float)r[e];
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            v[e] = 0.f;
            if (e < left) v[e] = (float)p[e];
        }
    }
}

template <class T, int VEC>
__device__ __forceinline__ void store_pack(T *__restrict__ p, int left, const float (&v)[VEC])
{
    if (left >= VEC) {
        typename Pack<T, VEC>::raw r;
#pragma unroll
        for (int e = 0; e < VEC; ++e) r[e] = (T)v[e];
        *reinterpret_cast<typename Pack<T, VEC>::type *>(p) = r;
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (e < left) p[e] = (T)v[e];
    }
}

// ---------------------------------------------------------------------------------------------
// host side: checks
// ---------------------------------------------------------------------------------------------
struct Extent { // bytes [lo, hi) from the first to the last element
    uintptr_t lo, hi;
    bool meets(const Extent &o) const { return lo < o.hi && o.lo < hi; }
};

inline size_t dtype_size(int dtype) { return dtype == SVGD_F32 ? 4 : 2; }

inline Extent extent(const svgd_rows &r, int dtype, int n, int64_t rows, int64_t width)
{
    const uintptr_t lo = (uintptr_t)r.data;
    const uintptr_t last = (uintptr_t)(n - 1) * (uintptr_t)r.particle_stride + (uintptr_t)(rows - 1) * (uintptr_t)r.row_stride + (uintptr_t)width;
    return {lo, lo + last * dtype_size(dtype)};
}
inline Extent extent(const float *p, int64_t stride, int n, int64_t size)
{
    return {(uintptr_t)p, (uintptr_t)p + ((uintptr_t)(n - 1) * (uintptr_t)stride + (uintptr_t)size) * 4};
}
inline Extent extent(const void *p, size_t bytes) { return {(uintptr_t)p, (uintptr_t)p + bytes}; }

// Strides and extents beyond this many elements are not those of memory; below it no offset leaves 64 bits.
constexpr int64_t kMaxStride = (int64_t)1 << 48;

inline int check_sizes(int dtype, int n, int64_t rows, int64_t width, int64_t max_width)
{
    if (dtype < SVGD_F32 || dtype > SVGD_F16 || n < 1 || rows < 0 || width < 1) return SVGD_ERR_INVALID_ARG;
    if (n > SVGD_MAX_PARTICLES || rows > SVGD_LAYER_MAX_ROWS || width > max_width) return SVGD_ERR_TOO_LARGE;
    return SVGD_OK;
}

inline bool aligned_to(const void *p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

inline bool valid_input(const svgd_rows &r, int dtype, int64_t rows)
{
    return r.data && aligned_to(r.data, dtype_size(dtype)) && r.particle_stride >= 0 && r.row_stride >= 0 && r.particle_stride <= kMaxStride &&
           (r.row_stride == 0 || rows <= kMaxStride / r.row_stride);
}

// An output's rows must not overlap: they lie particle by particle or row by row.
inline bool valid_output(const svgd_rows &r, int dtype, int n, int64_t rows, int64_t width)
{
    if (!valid_input(r, dtype, rows)) return false;
    const int64_t ps = r.particle_stride, rs = r.row_stride;
    if (n == 1) return rows == 1 || rs >= width;
    if (rows == 1) return ps >= width;
    return (rs >= width && ps >= (rows - 1) * rs + width) || (ps >= width && rs >= (n - 1) * ps + width);
}

// The particles' parts of a parameter: `size` floats every `stride`
struct Params {
    const float *p;
    int64_t stride, size;
};

inline bool valid_params(const Params &a, int n, bool output)
{
    return a.p && aligned_to(a.p, 4) && a.stride >= 0 && a.stride <= kMaxStride && (!output || n == 1 || a.stride >= a.size);
}

// Whether any particle's part of one meets any of the other's.  They mostly lie in the same rows, side by side: their
// extents meet, they do not.
inline bool params_meet(const Params &a, const Params &b, int n)
{
    if (!extent(a.p, a.stride, n, a.size).meets(extent(b.p, b.stride, n, b.size))) return false;
    if (a.stride == b.stride && a.stride > 0) {
        // part j of b starts d + (j - i) stride floats behind part i of a: the first j - i at which b's part does not end before a's
        const int64_t s = a.stride, d = ((intptr_t)b.p - (intptr_t)a.p) / 4, lo = -b.size - d; // m s > lo
        int64_t m = lo >= 0 ? lo / s + 1 : -((-lo - 1) / s);
        if (m < -(int64_t)(n - 1)) m = -(int64_t)(n - 1);
        return m <= n - 1 && d + m * s < a.size;
    }
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < n; ++j)
            if (extent(a.p + i * a.stride, 0, 1, a.size).meets(extent(b.p + j * b.stride, 0, 1, b.size))) return true;
    return false;
}

} // namespace svgd
