// Attention, forward, activations of type f32.
#define SVGD_ATTENTION_TYPE float
#include "attention_forward_instance.hpp"
