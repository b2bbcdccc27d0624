/*
 * svgd_layers.h - C ABI of the particles' own layers: layer norm, gated feed-forward block and dropout,
 * forward and backward, for all n networks of an ensemble at once.
 *
 * svgd_step (svgd.h) takes the parameters of n networks as the rows of X and their scores as the rows of G.
 * These calls are what a network makes its score with: a layer's parameters are read where they lie in the
 * rows of X and their gradients are written to the same places of G, so that nothing is packed, flattened
 * or copied between a backward pass and the step (paper App. B.2: the leader gathers every particle's
 * parameters and gradients into flat vectors).  The three together are the residual feed-forward half of a
 * transformer block, s = x + dropout(ffn(layer_norm(x))).
 *
 * Conventions for every entry point
 *   - Activations are n particles x `rows` x `width` values of one svgd_dtype in DEVICE memory, described by
 *     svgd_rows: value c of row t of particle i is element i * particle_stride + t * row_stride + c of
 *     `data`.  Inputs may have any strides (a particle stride of 0: all particles see the same rows).  Rows of
 *     outputs must not overlap.  Only the alignment of the type is required.
 *   - Parameters and their gradients are fp32 in DEVICE memory, particle i's at i * stride elements from the
 *     pointer (`stride` is the distance of two rows of X or G), contiguous and row-major within a particle.
 *     Only 4-byte alignment is required.
 *   - Sums, means, products and whatever else lies between the inputs and the outputs are held in fp32 (or
 *     more), whatever the activations' type; each output is rounded once.
 *   - `accumulate` 0: gradients of parameters are overwritten; otherwise they are added to what is there.
 *   - rows = 0 is allowed: nothing is read or written but gradients of parameters, which become (or stay as
 *     with `accumulate`) what a sum over no rows is.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  All work is enqueued on it, on the
 *     current device; calls do not synchronise or allocate and can be captured into a graph.  Scratch memory
 *     is the caller's; what a call leaves in it means nothing.  Results do not depend on what runs beside a call:
 *     the same inputs give the same bits.
 *   - Return value: SVGD_OK or a negative svgd_status: INVALID_ARG for null pointers, sizes below 1 (rows: 0),
 *     misaligned pointers, an unknown type or activation, outputs that overlap each other or an input, a
 *     non-finite eps or p outside [0, 1]; TOO_LARGE beyond the limits below.  Nothing is launched then.  DEVICE if a launch failed: those
 *     that the call made before it stay on the stream.  Tensors' extents count, from the first to the last of their elements, except
 *     where the parts of parameters and of their gradients lie side by side in the same rows: those are looked at one by one.
 *     No entry point aborts or throws.  Non-finite DATA is not checked and propagates as NaN or Inf.
 */
#ifndef SVGD_LAYERS_H
#define SVGD_LAYERS_H

#include <stddef.h>
#include <stdint.h>

#include "svgd.h"

#ifdef __cplusplus
extern "C" {
#endif

enum svgd_dtype { SVGD_F32 = 0, SVGD_BF16 = 1, SVGD_F16 = 2 };
enum svgd_activation { SVGD_SILU = 0, SVGD_GELU = 1 /* with the error function, no approximation */ };

typedef struct svgd_rows {
    void *data;
    int64_t particle_stride, row_stride; /* in elements */
} svgd_rows;

/* n <= SVGD_MAX_PARTICLES, and per particle: */
#define SVGD_LAYER_MAX_ROWS ((int64_t)1 << 30)
#define SVGD_LAYER_MAX_NORM 16384            /* width that svgd_layer_norm_* takes */
#define SVGD_LAYER_MAX_WIDTH ((int64_t)1 << 20) /* width and hidden width of svgd_gated_ffn_* */
/* (svgd_dropout takes rows of up to SVGD_MAX_D values; svgd_gated_ffn_* work in tiles, and those of a launch are below 2^24: of g, u and
 * their gradients, n ceil(rows / 128) ceil(hidden / 128) of them, of y and dx half as many by the width, of the parameters' gradients 3 n ceil(width / 256) ceil(hidden / 128)) */

/*
 * Layer norm over the values of each row:
 *     mean = avg_c x_c,  rstd = 1 / sqrt(avg_c (x_c - mean)^2 + eps),  y_c = (x_c - mean) rstd weight_c + bias_c
 * weight and bias: `width` values per particle; bias may be NULL.  mean and rstd (DEVICE, n * rows floats each,
 * particle-major) are what the backward pass needs, which takes them as they are, rounded to fp32; both may be NULL.
 */
int svgd_layer_norm_forward(int dtype, int n, int64_t rows, int64_t width, svgd_rows x, const float *weight,
                            int64_t weight_stride, const float *bias, int64_t bias_stride, double eps, svgd_rows y,
                            float *mean, float *rstd, void *stream);

/*
 * Its backward pass: with a = dy * weight and xhat = (x - mean) rstd,
 *     dx = rstd (a - avg_c a - xhat avg_c (a xhat)),  dweight = sum_t dy xhat,  dbias = sum_t dy
 * dx.data, dweight and dbias may be NULL: that gradient is not wanted then.  scratch (DEVICE, 16-byte aligned):
 * svgd_layer_norm_scratch bytes; may be NULL if neither dweight nor dbias is wanted.
 */
size_t svgd_layer_norm_scratch(int n, int64_t rows, int64_t width);
int svgd_layer_norm_backward(int dtype, int n, int64_t rows, int64_t width, svgd_rows dy, svgd_rows x,
                             const float *weight, int64_t weight_stride, const float *mean, const float *rstd,
                             svgd_rows dx, float *dweight, int64_t dweight_stride, float *dbias, int64_t dbias_stride,
                             int accumulate, void *scratch, size_t scratch_bytes, void *stream);

/*
 * Gated feed-forward block:
 *     g = gate x,  u = up x,  h = act(g) * u,  y = down h            for every row x
 * gate and up: hidden x width, down: width x hidden values per particle.  buffer (DEVICE, 16-byte
 * aligned, svgd_gated_ffn_buffer bytes) holds h during the call; with `save` it also receives g and u and is, as it
 * is afterwards, what the backward pass takes.  scratch (DEVICE, 16-byte aligned): svgd_gated_ffn_forward_scratch
 * bytes, may be NULL if these are 0.  Non-finite inputs make what depends on them non-finite, but an
 * infinity may come out as NaN, and so may what depends on finite fp32 values beyond 3.389e38 (the largest bf16 value).
 * Of factors below 1e-33 in size the products' accuracy falls off, by 1e-36 to some 1e-5 of them.
 */
size_t svgd_gated_ffn_buffer(int n, int64_t rows, int64_t width, int64_t hidden, int save);
size_t svgd_gated_ffn_forward_scratch(int n, int64_t rows, int64_t width, int64_t hidden);
int svgd_gated_ffn_forward(int dtype, int activation, int n, int64_t rows, int64_t width, int64_t hidden, svgd_rows x,
                           const float *gate, int64_t gate_stride, const float *up, int64_t up_stride,
                           const float *down, int64_t down_stride, svgd_rows y, int save, void *buffer,
                           size_t buffer_bytes, void *scratch, size_t scratch_bytes, void *stream);

/*
 * Its backward pass, `saved` being the buffer of the forward call with `save` (read only here):
 *     dh = dy down,  dg = dh u act'(g),  du = dh act(g)
 *     dx = dg gate + du up,  dgate = sum_t dg x^T,  dup = sum_t du x^T,  ddown = sum_t dy h^T
 * dx.data, and each of dgate, dup and ddown, may be NULL: that gradient is not wanted then (without any of the parameters'
 * dx may be summed up in another order: its last bits may be others).  scratch (DEVICE, 16-byte aligned): svgd_gated_ffn_scratch bytes.
 */
size_t svgd_gated_ffn_scratch(int n, int64_t rows, int64_t width, int64_t hidden);
int svgd_gated_ffn_backward(int dtype, int activation, int n, int64_t rows, int64_t width, int64_t hidden, svgd_rows dy,
                            svgd_rows x, const float *gate, int64_t gate_stride, const float *up, int64_t up_stride,
                            const float *down, int64_t down_stride, const void *saved, size_t saved_bytes, svgd_rows dx,
                            float *dgate, int64_t dgate_stride, float *dup, int64_t dup_stride, float *ddown,
                            int64_t ddown_stride, int accumulate, void *scratch, size_t scratch_bytes, void *stream);

/*
 * Dropout from the counter-based generator of this package's workloads; no mask is stored.  Value e (counted over
 * n x rows x width, the last fastest, whatever the strides) has the 32 random bits r_e: the upper (e even) or lower (e odd)
 * half of splitmix64(base + e / 2), base = splitmix64(splitmix64(seed) + call), where splitmix64(v) is that
 * generator's output for the state v.  With `counter` (DEVICE, one int64, 8-byte aligned) base is further replaced by
 * splitmix64(base + *counter) when the kernel runs: a replayed graph draws anew where the caller moves the counter on.
 *     keep_e = r_e >= round(p 2^32),   y_e = keep_e ? x_e / (1 - p) : 0,   plus residual_e if residual.data is not NULL
 * A dropped value counts as 0 whatever it is (NaN included); p = 1 drops all.  y may be x or the residual
 * itself (same pointer and strides).  The backward pass is the same call on dy without a residual (the residual's gradient
 * is dy): same p, seed, call and *counter.
 */
int svgd_dropout(int dtype, int n, int64_t rows, int64_t width, svgd_rows x, svgd_rows residual, svgd_rows y, double p,
                 uint64_t seed, uint64_t call, const int64_t *counter, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SVGD_LAYERS_H */
