// Attention, gradients of queries, activations of type bf16.
#define SVGD_ATTENTION_TYPE svgd::bf16_t
#include "attention_queries_instance.hpp"
