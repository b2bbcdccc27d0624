// Linear maps, activations of type bf16.
#define SVGD_LINEAR_TYPE svgd::bf16_t
#include "linear_instance.hpp"
