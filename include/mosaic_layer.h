/*
 * mosaic_layer.h -- C ABI of libmosaic, second part: the layer work on either side of the mask-only logits
 * (mosaic.h): root-mean-square norm with the residual's addition, activations kept in 8 bits, and the gated
 * feed-forward block, with their backward passes.  The final norm makes the `hidden` rows that the mask-only pass reads,
 * for the masked positions alone; the feed-forward activations are the other memory peak of a denoising step
 * (paper section 3, observation 3, and section 4.4), which the block here does not write.
 *
 * The conventions of mosaic.h hold: device pointers owned by the caller, `stream` a hipStream_t (NULL = the default
 * stream), calls only enqueue, allocate nothing and keep nothing; argument errors are found before anything is enqueued.
 * Matrices are row-major with dense rows; ld_* is the distance of two rows in elements.
 *   bf16 and 32-bit matrices: base 16-byte aligned, ld_* a multiple of 8, at most 2^21
 *   an output overlaps an input only where that is said to be allowed
 *   every sum over a row, a column or a product is held in 32 bits; a result is rounded to its type once.  The exception is
 *   said at mosaic_gated_ffn_backward
 * T = rows (positions; 0 <= T < 2^31; T == 0 enqueues nothing but the clearing of sums over rows), d = hidden size,
 * F = feed-forward size; d and F are multiples of 8, at most MOSAIC_MAX_ROW (the norms, the checkpoints and what works from
 * 8-bit rows: d at most MOSAIC_MAX_NORM_ROW).  A workspace query gives 0 for sizes that its call refuses.
 * Results do not depend on anything but the arguments: no atomics, the same bits on every call.  A row's norm, its gradient and its
 * 8 bits are the same whatever other rows the call has.  The feed-forward block sums a product's K in an order that follows
 * from the sizes, T among them: the same rows in calls of another number of rows may differ in their last bits.
 */
#ifndef MOSAIC_LAYER_H_
#define MOSAIC_LAYER_H_

#include "mosaic.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MOSAIC_MAX_NORM_ROW 16384
#define MOSAIC_MAX_ROW (1 << 17)

/* Element types of the arguments that may have either. */
typedef enum { MOSAIC_BF16 = 0, MOSAIC_F32 = 1 } mosaic_type;

/* 8-bit formats: int8 in -127..127; e4m3 (OCP: 4 exponent, 3 fraction bits, no infinity) in -448..448. */
typedef enum { MOSAIC_INT8 = 0, MOSAIC_E4M3 = 1 } mosaic_q8_format;

/* Activations of the gated feed-forward block: g / (1 + exp(-g)), and the tanh form of the Gaussian error unit
 * g/2 (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))). */
typedef enum { MOSAIC_SILU = 0, MOSAIC_GELU_TANH = 1 } mosaic_activation;

/*
 * A [T, d] matrix in 8 bits: per row, every `group` consecutive columns share a scale (the last group may be shorter).
 *   scale = a / top, a = the largest magnitude of the group, top = 127 (int8) or 448 (e4m3)
 *   value = v * (top / a) rounded to the nearest number of the format, ties to even
 * and the element stands for bf16(value * scale).  A group whose a is below 2^-112 is stored as zeros with scale 0; one
 * that holds a NaN or an infinity gets scale NaN and values 0, so all of it is restored as NaN.
 *   values   dev, 1 byte each, 8-byte aligned, ld_values a multiple of 8
 *   scales   dev float [T, ld_scales], ld_scales >= ceil(d / group)
 *   group    32, 64 or 128
 */
typedef struct {
  void *values;
  float *scales;
  int64_t ld_values;
  int64_t ld_scales;
  int32_t format;
  int32_t group;
} mosaic_q8_rows;

/*
 * Stores rows in 8 bits, and restores them.
 *   x / out   bf16 or 32-bit [T, d] by `type`
 */
int mosaic_checkpoint_store(const void *x, int32_t type, int64_t ld_x, int64_t T, int32_t d, const mosaic_q8_rows *q8,
                            void *stream);
int mosaic_checkpoint_load(const mosaic_q8_rows *q8, int64_t T, int32_t d, void *out, int32_t type, int64_t ld_out,
                           void *stream);

/*
 * Root-mean-square norm with the residual's addition, per row t:
 *   h = x + residual                          (either may be NULL, not both: then h is the other one)
 *   y = h / sqrt(mean(h^2) + eps) * gamma     (from the sum in 32 bits, before it is rounded to its type)
 * Outputs, each optional but not all absent: sum = h, y, and y in 8 bits (from y in 32 bits).
 *   x          bf16 [T, d]; residual, sum: bf16 or 32-bit by `stream_type`; sum may be the residual's own memory
 *   gamma      [d], bf16 or 32-bit by `gamma_type`, 16-byte aligned
 *   y          bf16 [T, d]; may be x's own memory
 *   eps        finite, > 0
 *   idx, count NULL for all rows; else only rows idx[0 .. *count) (dev int32, as mosaic_mask_compact makes them, at
 *              most max_rows of them, no row twice) are read and written, the rest is untouched; an entry outside
 *              [0, T) is skipped
 *   q8         host pointer or NULL
 * A NaN makes its row NaN, an infinity its own element (the rest of the row is zero); other rows are not affected.  Squares are
 * summed in 32 bits: a row whose sum of squares passes 3e38 counts as infinite.
 */
int mosaic_rmsnorm_forward(const void *x, int64_t ld_x, const void *residual, int32_t stream_type, int64_t ld_residual,
                           const void *gamma, int32_t gamma_type, float eps, int64_t T, int32_t d, const int32_t *idx,
                           const int32_t *count, int64_t max_rows, void *sum, int64_t ld_sum, void *y, int64_t ld_y,
                           const mosaic_q8_rows *q8, void *stream);

/*
 * Its gradient at h.  With n = h / sqrt(mean(h^2) + eps), c = gamma * dy:
 *   dsum    = (c - n * mean(c * n)) / sqrt(mean(h^2) + eps)  [+ dsum_in]
 *   dgamma  = sum over the rows of dy * n          [+ what dgamma holds, if accumulate]
 * x and residual both have the gradient dsum.
 *   dy         bf16 [T, d]
 *   h          what the forward pass kept of the sum: bf16 or 32-bit by `stream_type`, or NULL and
 *   q8         its rows in 8 bits
 *   dsum_in    gradient that reaches the sum past the norm, or NULL; it and dsum by `stream_type`; dsum may be
 *              dsum_in's own memory, or NULL where only dgamma is wanted
 *   dgamma     float [d], or NULL
 *   workspace  dev, 16-byte aligned, mosaic_rmsnorm_backward_workspace_bytes(T, d) bytes (needed only for dgamma)
 */
int64_t mosaic_rmsnorm_backward_workspace_bytes(int64_t T, int32_t d);
int mosaic_rmsnorm_backward(const void *dy, int64_t ld_dy, const void *h, int64_t ld_h, const mosaic_q8_rows *q8,
                            int32_t stream_type, const void *gamma, int32_t gamma_type, float eps, int64_t T, int32_t d,
                            const void *dsum_in, int64_t ld_dsum_in, void *dsum, int64_t ld_dsum, float *dgamma,
                            int32_t accumulate, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * Gated feed-forward block up to the down projection, in one kernel; neither projection is ever written:
 *   out = act(x w_gate^T) * (x w_up^T)
 *   x       bf16 [T, d];  w_gate, w_up: bf16 [F, d], row stride ld_w (two halves of one packed matrix are fine)
 *   out     bf16 [T, F]
 */
int mosaic_gated_ffn_forward(const void *x, int64_t ld_x, const void *w_gate, const void *w_up, int64_t ld_w, int64_t T,
                             int32_t d, int32_t F, int32_t activation, void *out, int64_t ld_out, void *stream);

/*
 * Its gradients, from the gradient of `out` and the block's input alone: both projections are computed again.  With
 * g = x w_gate^T, u = x w_up^T:
 *   dg = dout * u * act'(g),  du = dout * act(g)      rounded to bf16, for the matrix cores (up to 2^-8 relative
 *                                                     per term, as for the results; in the 2-norm of a result of
 *                                                     many terms 0.0023 in all, where its own rounding is 0.0017);
 *                                                     up to 32 rows with what that leaves over in a second number
 *                                                     each, so that the results' own rounding is all there is
 *   dx = dg w_gate + du w_up,   dw_gate = dg^T x,   dw_up = du^T x
 *   x          bf16 [T, d], or NULL and
 *   q8         its rows in 8 bits; the gradients are those at the values they stand for
 *   dout       bf16 [T, F]
 *   out        NULL, or bf16 [T, F]: the block's output again (for the down projection's gradient)
 *   dx         bf16 [T, d] or NULL
 *   dw_gate, dw_up   both or neither NULL; [F, d] bf16 or 32-bit by `dw_type`, row stride ld_dw
 *   accumulate nonzero: the weight gradients are added to what dw_gate and dw_up hold (32-bit only), so that a batch can be
 *              taken in parts
 *   workspace  dev, 16-byte aligned, mosaic_gated_ffn_backward_workspace_bytes(T, d, F, q8 != NULL) bytes: dg and du,
 *              4 T F bytes (up to 32 rows 8 T F), the restored input, 2 T d, and for up to 4096 rows partial sums of dx.  A
 *              workspace for T rows serves fewer rows, too
 */
int64_t mosaic_gated_ffn_backward_workspace_bytes(int64_t T, int32_t d, int32_t F, int32_t q8_input);
int mosaic_gated_ffn_backward(const void *dout, int64_t ld_dout, const void *x, int64_t ld_x, const mosaic_q8_rows *q8,
                              const void *w_gate, const void *w_up, int64_t ld_w, int64_t T, int32_t d, int32_t F,
                              int32_t activation, void *out, int64_t ld_out, void *dx, int64_t ld_dx, void *dw_gate,
                              void *dw_up, int32_t dw_type, int64_t ld_dw, int32_t accumulate, void *workspace,
                              int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MOSAIC_LAYER_H_ */
