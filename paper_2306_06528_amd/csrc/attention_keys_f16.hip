// Attention, gradients of keys and values, activations of type f16.
#define SVGD_ATTENTION_TYPE svgd::f16_t
#include "attention_keys_instance.hpp"
