/*
 * mosaic_tokens.h -- C ABI of libmosaic, third part: both ends of a masked-diffusion model, for training and for scoring.
 * Tokens into rows (embedding lookup with scaling, dropout) and rows back onto given tokens (log probabilities at the
 * masked positions, with entropy and the most probable alternatives), with their backward passes.  The mask-only pass of
 * mosaic.h answers which token a masked position takes; the calls here say how probable a given one is there, which is what
 * the training loss, a likelihood and the confidences by margin and by entropy are made of, and, like that pass, never
 * write a row's logits.
 *
 * The conventions of mosaic.h and mosaic_layer.h hold: device pointers owned by the caller, `stream` a hipStream_t (NULL = the
 * default stream), calls only enqueue, allocate nothing and keep nothing; argument errors are found before anything is
 * enqueued; a workspace query gives 0 for sizes that its call refuses.  Matrices are row-major with dense rows, base 16-byte
 * aligned, ld_* the distance of two rows in elements, a multiple of 8, at most 2^21; an output overlaps an input only where
 * that is said to be allowed.  Types are mosaic_type's.
 * T = positions (0 <= T < 2^31), V = vocabulary size (1 <= V < 2^31 - 256), d = hidden size, a multiple of 8, at most
 * MOSAIC_MAX_ROW.  Sums and statistics are held in 32 bits, a result is rounded to its type once.
 * No atomics on floating-point numbers: the same bits on every call of the same arguments.
 */
#ifndef MOSAIC_TOKENS_H_
#define MOSAIC_TOKENS_H_

#include "mosaic_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Embedding lookup: out[t] = scale * table[tokens[t]] for t < T; a row of zeros where tokens[t] lies outside [0, V)
 * (a padding position).
 *   tokens     dev int32[T]
 *   count      dev int32[1] or NULL: only the first min(*count, T) rows are written, the rest are left as they were
 *   table      [V, d], bf16 or 32-bit by `table_type`; only rows that tokens name are read
 *   scale      finite
 *   out        [T, d], bf16 or 32-bit by `out_type`
 * With hidden states as the table and a gather list as the tokens, it gathers rows.
 */
int mosaic_embedding_forward(const int32_t *tokens, int64_t T, const int32_t *count, const void *table, int32_t table_type,
                             int64_t ld_table, int32_t V, int32_t d, float scale, void *out, int32_t out_type,
                             int64_t ld_out, void *stream);

/*
 * Its gradient: dtable[v] = scale * (sum of dout[t] over the t with tokens[t] == v)  [+ what dtable[v] holds, if accumulate].
 * Tokens are sorted, stably, and a row of the table is summed in the order of its positions; a token of many positions (half
 * of them are [MASK]) in parts that are joined in order.  Where the parts end follows from all of the tokens: a row's last
 * bits may depend on the tokens beside it.
 *   dout       [T, d], bf16 or 32-bit by `dout_type`
 *   tokens, count   as above; rows from *count on and tokens outside [0, V) have no part in it
 *   dtable     [V, d], bf16 or 32-bit by `dtable_type`.  Without accumulate every row is written (zeros where no token names
 *              it); with it (32-bit only) rows that no token names are left as they were
 *   workspace  dev, 16-byte aligned, mosaic_embedding_backward_workspace_bytes(T, d, V) bytes
 * With a gather list as the tokens and V = the rows of the hidden states it brings the gradients of gathered rows back,
 * also where a row is listed twice (mosaic_shift_indices).
 */
int64_t mosaic_embedding_backward_workspace_bytes(int64_t T, int32_t d, int32_t V);
int mosaic_embedding_backward(const void *dout, int32_t dout_type, int64_t ld_dout, const int32_t *tokens, int64_t T,
                              const int32_t *count, int32_t V, int32_t d, float scale, void *dtable, int32_t dtable_type,
                              int64_t ld_dtable, int32_t accumulate, void *workspace, int64_t workspace_bytes,
                              void *stream);

/*
 * Dropout whose mask is never stored: it follows from the seed, the element's row and column, and which dropout of the model
 * it is, so that the backward pass, or a forward pass taken again, makes the same one.
 *   border   = p * 2^16, rounded
 *   r(t, c)  = 16 bits of Philox4x32-10 (Salmon et al., SC'11) with key = (low, high 32 bits of seed) and counter =
 *              (c / 8, low and high 32 bits of first_row + t, site + 1): of output word c / 2 % 4 the low half where c is even,
 *              else the high half
 *   keep     = r >= border
 *   forward  out = (keep ? x * 2^16 / (2^16 - border) : 0)  [+ residual]       from 32 bits, rounded once
 *   backward dx  = keep ? dout * 2^16 / (2^16 - border) : 0
 * The factor belongs to the share that is dropped in fact, border / 2^16, so the mean is kept.  A dropped element is 0 (or the
 * residual) whatever x holds there, a NaN too.
 *   x          bf16 [T, d];  residual ([T, d] or NULL) and out: bf16 or 32-bit by `stream_type`
 *   dout       [T, d], bf16 or 32-bit by `stream_type`;  dx: bf16 [T, d]
 *   p          0 <= p <= 1 - 2^-16
 *   site       0 <= site < 2^31 - 1
 *   first_row  >= 0: number of the first row, so that a batch can be taken in parts
 * out may be the residual's own memory, and x's where stream_type is MOSAIC_BF16; dx may be dout's where that is MOSAIC_BF16
 * (with the same row stride).
 */
int mosaic_dropout_forward(const void *x, int64_t ld_x, const void *residual, int32_t stream_type, int64_t ld_residual,
                           int64_t T, int32_t d, float p, uint64_t seed, int32_t site, int64_t first_row, void *out,
                           int64_t ld_out, void *stream);
int mosaic_dropout_backward(const void *dout, int32_t stream_type, int64_t ld_dout, int64_t T, int32_t d, float p,
                            uint64_t seed, int32_t site, int64_t first_row, void *dx, int64_t ld_dx, void *stream);

/*
 * Log probabilities of given tokens at listed rows, with the entropy of a row's distribution and its most probable
 * alternatives; no logits are written.  For every j < M = min(*count, max_rows), with h = hidden[idx[j]]:
 *   x[v]           = sum_k h[k] * w[v, k]              bf16 x bf16, 32-bit sums, no bias
 *   out_lse[j]     = log sum_v exp(x[v])
 *   out_logprob[j] = x[targets[j]] - out_lse[j];  0 where targets[j] lies outside [0, V) (a row without a target)
 *   out_entropy[j] = - sum_v p[v] log p[v],  p[v] = exp(x[v] - out_lse[j])
 *   top_id[j, i], top_logprob[j, i], i < n_top:  the ids with the largest logits, the lower id first among equals, and
 *                    x[id] - out_lse[j];  -1 and -infinity past the vocabulary
 *   hidden     bf16 [T, d];  w: bf16 [V, d]
 *   idx, count dev int32, as mosaic_mask_compact makes them, or both NULL for all rows (then max_rows = T).  Rows may be listed
 *              in any order and more than once; an entry outside [0, T) is clamped to it
 *   max_rows   bound on *count, at most 2^31 - 256.  What the call takes follows from the rows found; its workspace from the bound
 *   targets    dev int32[max_rows], of the listed rows in their order; needed for out_logprob alone
 *   out_*      dev float[max_rows], each may be NULL, not all of them with n_top = 0; entries from M on are left as they were
 *   n_top      0 .. MOSAIC_MAX_TOP;  top_id int32 and top_logprob float [max_rows, n_top], dense, NULL where it is 0
 *   workspace  dev, 16-byte aligned, mosaic_masked_logprobs_workspace_bytes bytes (one for more rows serves fewer): sums of the
 *              vocabulary's parts, with alternatives lists of their candidates (67 MB) and the parts' best, and, where the
 *              hidden states pass 2 GiB, the listed rows side by side (counted without a list, too, and not used then)
 * A NaN among a row's logits makes that row's log probabilities, entropy and log-sum-exp NaN and its alternatives unspecified
 * (ids in [-1, V)), an infinite one (of infinite weights or states; 2^100 and more counts as one) at least its entropy; other rows
 * are not affected.
 * How the vocabulary is parted follows from the rows found: a row's last bits may depend on their number.
 */
#define MOSAIC_MAX_TOP 16
int64_t mosaic_masked_logprobs_workspace_bytes(int64_t T, int64_t ld_h, int64_t max_rows, int32_t d, int32_t V, int32_t n_top);
int mosaic_masked_logprobs(const void *hidden, int64_t ld_h, int64_t T, int32_t d, const void *w, int64_t ld_w, int32_t V,
                           const int32_t *idx, const int32_t *count, int64_t max_rows, const int32_t *targets,
                           float *out_logprob, float *out_entropy, float *out_lse, int32_t n_top, int32_t *top_id,
                           float *top_logprob, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * Its gradients, from those of out_logprob (g) and out_entropy (h); the logits are computed again, a part of the vocabulary at a
 * time.  With p[j, v] and the entropy H[j] as above:
 *   dl[j, v] = g[j] ([v == targets[j]] - p[j, v]) - h[j] p[j, v] (log p[j, v] + H[j])       (g[j] = 0 without a target)
 *   dx[j]    = sum_v dl[j, v] w[v]                              the gradient at the listed row hidden[idx[j]]
 *   dw[v]    = sum_j dl[j, v] hidden[idx[j]]                    [+ what dw holds, if accumulate]
 * dl is rounded to bf16 for the matrix cores (up to 2^-8 relative per term), with what that leaves over in a second number
 * each (2^-16 then) where dw has 32 bits, for dw, and where max_rows is 32 or less, for both results.  The target's entries,
 * which outweigh the others, go into both sums in 32 bits.
 *   hidden .. targets   as for the forward pass
 *   logprob, entropy, lse   dev float[max_rows], what the forward pass gave: lse always, logprob with dlogprob, entropy with dentropy
 *   dlogprob   dev float[max_rows], or NULL (then targets and logprob are not looked at);  dentropy: the same, or NULL; not both NULL
 *   dx         bf16 [max_rows, d] or NULL; rows from M on are left as they were.  A program whose listed rows are all different
 *              scatters them itself; mosaic_embedding_backward with idx as the tokens does it also where they are not.  Of an entry
 *              outside [0, T), clamped here as in the forward pass, it takes no gradient: such a list is clamped by the caller
 *   dw         [V, d] by `dw_type`, row stride ld_dw, or NULL; not both NULL.  Every row is written
 *   accumulate nonzero: dw is added to (32-bit only), so that a batch can be taken in parts
 *   workspace  dev, 16-byte aligned: the listed rows twice, 32-bit sums of dx, the targets' terms of dw (4 max_rows d bytes each and
 *              more for few rows), and dl of as many ids as the rest holds, 2 max_rows bytes each, with second numbers 4, of these at
 *              least 256.  The query answers for at most budget_bytes where that is enough, 0 or less: dl of up to 256 MiB; one for more
 *              rows serves fewer.  The sums' last bits follow from the size, and from whether there are second numbers
 * Every row of the bound costs what a listed one does: a close max_rows is worth its while.
 */
int64_t mosaic_masked_logprobs_backward_workspace_bytes(int64_t max_rows, int32_t d, int32_t V, int64_t budget_bytes);
int mosaic_masked_logprobs_backward(const void *hidden, int64_t ld_h, int64_t T, int32_t d, const void *w, int64_t ld_w, int32_t V,
                                    const int32_t *idx, const int32_t *count, int64_t max_rows, const int32_t *targets,
                                    const float *logprob, const float *entropy, const float *lse, const float *dlogprob,
                                    const float *dentropy, void *dx, int64_t ld_dx, void *dw, int32_t dw_type, int64_t ld_dw,
                                    int32_t accumulate, void *workspace, int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MOSAIC_TOKENS_H_ */
