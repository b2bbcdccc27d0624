// Attention, gradients of keys and values, activations of type f32.
#define SVGD_ATTENTION_TYPE float
#include "attention_keys_instance.hpp"
