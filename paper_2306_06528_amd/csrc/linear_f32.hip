// Linear maps, activations of type f32.
#define SVGD_LINEAR_TYPE float
#include "linear_instance.hpp"
