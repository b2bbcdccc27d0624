// The launches of both passes, by the plan that linear_rules.hpp makes.  The kernels' instances are compiled type by type
// (linear_<type>.hip).
#pragma once
#include "ffn_launch.hpp"
#include "linear_kernels.hpp"

namespace svgd {

struct LinearCall {
    LinearShape s;
    Params weight, bias, dweight, dbias;
    svgd_rows x, y, residual, dy, dx;
    float *z, *scratch;
    bool accumulate;
    hipStream_t stream;
};

template <class T> int linear_forward(const LinearCall &c, const LinearForwardPlan &plan);
template <class T> int linear_backward(const LinearCall &c, const LinearBackwardPlan &plan);

} // namespace svgd
