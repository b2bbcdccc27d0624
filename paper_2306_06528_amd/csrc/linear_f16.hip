// Linear maps, activations of type f16.
#define SVGD_LINEAR_TYPE svgd::f16_t
#include "linear_instance.hpp"
