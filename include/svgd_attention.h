/*
 * svgd_attention.h - C ABI of the attention half of the particles' layers: linear maps with bias, activation and residual, norms of
 * queries and keys with the rotation by their positions, and attention, forward and backward, for all n networks of an ensemble at once.
 *
 * With the calls of svgd_layers.h these make whole transformer blocks of n networks: s = s +
 * linear(attention(rotary(linear(layer_norm(s))))), then the gated feed-forward half.
 *
 * Conventions: those of svgd_layers.h (activations of one svgd_dtype, parameters fp32 in the rows of X, their gradients in G, sums,
 * products and softmax statistics in fp32 or more - 16-bit attention's probabilities and gradients of scores, once they are operands of a
 * product, in two parts of the activations' type, 2^-17 of bf16 ones and 2^-22 of fp16 ones -, `accumulate`, `stream`, status, no
 * synchronisation or allocation, the same inputs give the same bits), and for activations with heads
 *   - n particles x `batch` sequences x `length` tokens x `heads` heads x `dim` values, described by svgd_heads: value c of head h of
 *     token t of sequence b of particle i is element i * particle_stride + b * batch_stride + t * token_stride + h * head_stride + c of
 *     `data`.  Inputs may have any strides from 0 on, a view into the results of one linear map among them; outputs' heads must not
 *     overlap, nor any other argument's values.  Two tensors whose addresses go through each other pass if their outer dimensions are
 *     the same and what is inside of these lies side by side: dq, dk and dv as the parts of one gradient of q, k and v together.
 */
#ifndef SVGD_ATTENTION_H
#define SVGD_ATTENTION_H

#include "svgd_layers.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Activations of svgd_linear_*; SVGD_SILU and SVGD_GELU among them. */
enum svgd_linear_activation { SVGD_RELU = 2, SVGD_TANH = 3, SVGD_NO_ACTIVATION = 4 };

typedef struct svgd_heads {
    void *data;
    int64_t particle_stride, batch_stride, token_stride, head_stride; /* in elements */
} svgd_heads;

#define SVGD_ATTENTION_MAX_DIM 128                   /* values of a head */
#define SVGD_ATTENTION_MAX_LENGTH ((int64_t)1 << 24) /* tokens and keys of a sequence, and tokens times heads that share keys */
#define SVGD_ATTENTION_MAX_BATCH ((int64_t)1 << 20)  /* sequences per particle; n batch heads length is below 2^28 - 16 too, and n batch kv_heads times the tiles of 64 keys, or rows, below 2^24 - 8 */
#define SVGD_ATTENTION_MAX_HEADS 4096
#define SVGD_ATTENTION_MAX_GROUP 256                 /* query heads to a key head */
#define SVGD_ATTENTION_MAX_STRIDE ((int64_t)1 << 23) /* of tokens, and of all the query heads to a key head, of q, k, v and do: less than this */
#define SVGD_ROTARY_MAX_DIM 256                      /* values of a head that svgd_qk_norm_rotary_* take */

/*
 * Linear map:
 *     z = weight x + bias,  y = act(z) + residual         for every row x
 * weight: out x width, bias: out values per particle; bias and residual.data may be NULL.  z (DEVICE, 16-byte aligned, svgd_linear_saved
 * bytes) receives z for the backward pass, which needs it unless the activation is none; may be NULL.  scratch (DEVICE, 16-byte aligned):
 * svgd_linear_forward_scratch bytes, may be NULL if these are 0.
 * Of non-finite and of very small factors the same holds as of svgd_gated_ffn_*.
 */
size_t svgd_linear_saved(int n, int64_t rows, int64_t out);
size_t svgd_linear_forward_scratch(int n, int64_t rows, int64_t width, int64_t out);
int svgd_linear_forward(int dtype, int activation, int n, int64_t rows, int64_t width, int64_t out, svgd_rows x, const float *weight,
                        int64_t weight_stride, const float *bias, int64_t bias_stride, svgd_rows residual, svgd_rows y, void *z,
                        size_t z_bytes, void *scratch, size_t scratch_bytes, void *stream);

/*
 * Its backward pass:
 *     dz = dy act'(z),  dx = dz weight,  dweight = sum_t dz x^T,  dbias = sum_t dz
 * The residual's gradient is dy.  dx.data, dweight and dbias may be NULL: that gradient is not wanted then.  scratch (DEVICE, 16-byte
 * aligned): svgd_linear_scratch bytes; svgd_linear_saved bytes less without an activation, where dz is dy.
 */
size_t svgd_linear_scratch(int n, int64_t rows, int64_t width, int64_t out);
int svgd_linear_backward(int dtype, int activation, int n, int64_t rows, int64_t width, int64_t out, svgd_rows dy, svgd_rows x,
                         const float *weight, int64_t weight_stride, const void *z, size_t z_bytes, svgd_rows dx, float *dweight,
                         int64_t dweight_stride, float *dbias, int64_t dbias_stride, int accumulate, void *scratch, size_t scratch_bytes,
                         void *stream);

/*
 * Norms of queries and keys, head by head, and the rotation by position, in one pass:
 *     y_c = x_c weight_c / sqrt(avg_c x_c^2 + eps),  pairs j of the first 2 `pairs` values of y turned by the angle position frequency_j
 * Pair j is the values j and j + pairs (interleaved = 0) or 2 j and 2 j + 1.  weights: `dim` values per particle, of queries and of keys;
 * either both or neither is NULL: no norm then.  frequencies (DEVICE, `pairs` doubles) and positions (DEVICE, int64 each; sequence b's
 * token t has positions[b * positions_stride + t], a stride of 0: all sequences the same) may be NULL if pairs is 0.  Angles are formed and
 * reduced in 64 bits.  heads or kv_heads may be 0 (q or k is not there).
 */
typedef struct svgd_rotary {
    int n, heads, kv_heads, dim, pairs, interleaved;
    int64_t batch, length;
    const double *frequencies;
    const int64_t *positions;
    int64_t positions_stride;
    double eps;
    const float *q_weight, *k_weight;
    int64_t q_weight_stride, k_weight_stride;
} svgd_rotary;
int svgd_qk_norm_rotary_forward(int dtype, const svgd_rotary *p, svgd_heads q, svgd_heads k, svgd_heads q_out, svgd_heads k_out, void *stream);

/*
 * Its backward pass, from q and k as the forward call got them (without a norm they are not read and may be NULL): with g = dy turned back,
 * xhat = x rstd and a = g weight,
 *     dx = rstd (a - xhat avg_c(a xhat)),  dweight = sum over sequences, tokens and heads of g xhat
 * dweights may be NULL, each for itself.  scratch (DEVICE, 16-byte aligned): svgd_qk_norm_rotary_scratch bytes; may be NULL if no dweight
 * is wanted.
 */
size_t svgd_qk_norm_rotary_scratch(const svgd_rotary *p);
int svgd_qk_norm_rotary_backward(int dtype, const svgd_rotary *p, svgd_heads dq_out, svgd_heads dk_out, svgd_heads q, svgd_heads k, svgd_heads dq,
                                 svgd_heads dk, float *dq_weight, int64_t dq_weight_stride, float *dk_weight, int64_t dk_weight_stride,
                                 int accumulate, void *scratch, size_t scratch_bytes, void *stream);

/*
 * Attention of `length` queries over `keys` keys of each sequence, heads / kv_heads query heads to a key head:
 *     z = scale q k;  z = cap tanh(z / cap) if cap > 0;  z -= slope |p - j| if slopes;  P = softmax of z over the keys that are seen;  o = P v
 * Query i is at position p = starts[b] + i (starts NULL: keys - length + i), key j at position j.  Query i sees key j where
 *     j < lengths[b] (NULL: keys), and not causal or j <= p or j < prefix[b] (NULL: 0), and documents[b, p] = documents[b, j] (NULL: all one)
 * A query whose position has no document (p < 0 or p >= keys) sees nothing if there are documents.  Where a query sees nothing o is 0 and
 * lse -infinity, and nothing flows back, whatever it and its d_o hold.  Keys and values from lengths[b] on are not read.  Those before it
 * have to be finite, seen or not: a non-finite one may make NaN of all of that head's results.  starts beyond +-2^28 count as that.
 * slopes: `heads` values per particle.  lse (DEVICE, n x batch x heads x length floats): log of the sum of exp z, for the backward pass;
 * may be NULL.  scratch (DEVICE, 16-byte aligned): svgd_attention_forward_scratch bytes of this same struct, may be NULL if these are 0.
 * Of non-finite and of very small fp32 factors the same holds as of svgd_gated_ffn_*.
 */
typedef struct svgd_attention {
    int n, heads, kv_heads, dim;
    int64_t batch, length, keys;
    int causal;
    double scale, cap; /* scale and cap from 1e-30 to 2e38, scale / cap from 2^-126 to 3e38; cap 0: none */
    const float *slopes;
    int64_t slopes_stride;
    const int32_t *starts, *lengths, *documents, *prefix; /* DEVICE: batch, batch, batch x keys, batch values */
} svgd_attention;
size_t svgd_attention_forward_scratch(const svgd_attention *a);
int svgd_attention_forward(int dtype, const svgd_attention *a, svgd_heads q, svgd_heads k, svgd_heads v, svgd_heads o, float *lse, void *scratch,
                           size_t scratch_bytes, void *stream);

/*
 * Its backward pass, o and lse being the forward call's: with dP = do v and dz = P (dP - sum_c do_c o_c),
 *     dslope = -sum dz |p - j|,  dz *= 1 - tanh^2,  dq = scale dz k,  dk = scale sum dz q,  dv = sum P do
 * dslopes (`heads` values per particle) may be NULL; with `accumulate` it is added to.  Gradients of keys that no query sees are 0.
 * scratch (DEVICE, 16-byte aligned): svgd_attention_scratch bytes.
 */
size_t svgd_attention_scratch(const svgd_attention *a);
int svgd_attention_backward(int dtype, const svgd_attention *a, svgd_heads d_o, svgd_heads q, svgd_heads k, svgd_heads v, svgd_heads o, const float *lse,
                            svgd_heads dq, svgd_heads dk, svgd_heads dv, float *dslopes, int64_t dslopes_stride, int accumulate, void *scratch,
                            size_t scratch_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SVGD_ATTENTION_H */
