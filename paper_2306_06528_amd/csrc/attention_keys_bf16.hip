// Attention, gradients of keys and values, activations of type bf16.
#define SVGD_ATTENTION_TYPE svgd::bf16_t
#include "attention_keys_instance.hpp"
