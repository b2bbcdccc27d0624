// Attention, gradients of queries, activations of type f16.
#define SVGD_ATTENTION_TYPE svgd::f16_t
#include "attention_queries_instance.hpp"
