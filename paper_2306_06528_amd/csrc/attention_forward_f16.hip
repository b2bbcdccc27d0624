// Attention, forward, activations of type f16.
#define SVGD_ATTENTION_TYPE svgd::f16_t
#include "attention_forward_instance.hpp"
