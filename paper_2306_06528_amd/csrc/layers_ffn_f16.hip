// Instances of the gated feed-forward block, fp16 activations.
#define SVGD_FFN_TYPE
#include "ffn_launch.hpp"

template int svgd::ffn_forward<svgd::f16_t>(const svgd::FfnCall &, const svgd::ForwardPlan &, const svgd_rows &, const svgd_rows &, float *, bool, float *);
template int svgd::ffn_backward<svgd::f16_t>(const svgd::FfnCall &, const svgd::BackwardPlan &, const svgd_rows &, const svgd_rows &, const float *, const svgd_rows &, const svgd::Params &,
                                     const svgd::Params &, const svgd::Params &, bool, float *);
