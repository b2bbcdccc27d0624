// Attention, gradients of queries, activations of type f32.
#define SVGD_ATTENTION_TYPE float
#include "attention_queries_instance.hpp"
