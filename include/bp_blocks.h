/*
 * bp_blocks.h -- C ABI of libbp.so, third part: what stands around the layers of
 * bp_experts.h in a model of blocks.
 *
 *   Embedding  rows of a table by token, and the pooled change of every token's row
 *              (a layer whose input is one unit out of many);
 *   Residual   the stream between blocks: a block's output is normed, gated, scaled and
 *              added, and the sum is normed again for the next block;
 *   Clip       the norm of many changes together, and the changes scaled down to a bound.
 *
 * The conventions of bp.h and bp_experts.h hold (row-major contiguous buffers, caller-owned device
 * memory, streams, status codes, bp_last_error; values float32 or bfloat16 as the handle's dtype says;
 * gates, norms' weights, biases, statistics and every change G float32 in both; BP_BF16 rows are
 * multiples of 8 units on 16-byte boundaries, and so is d_G of their embeddings; other float32 and int
 * buffers lie on 4-byte boundaries).  Values
 * are computed and summed in float32 and rounded once, on the way out.  Besides:
 *   - A handle belongs to the device that was current when it was made; calls with another
 *     one current are refused (BP_EINVAL).
 *   - Handles own scratch that each call reuses: calls on one handle, and graphs captured from
 *     them, belong on one stream at a time.  Compute calls allocate nothing and may be captured.
 *   - A call has the same bits on every run: the order of its sums depends on its sizes, ids and offsets, on whether
 *     its float32 buffers lie on 16-byte boundaries, and on the device's number of SMs, and on nothing else.
 */
#ifndef BP_BLOCKS_H
#define BP_BLOCKS_H

#include "bp.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct bp_embedding bp_embedding;
typedef struct bp_residual bp_residual;
typedef struct bp_clip bp_clip;

#define BP_MAX_TOKENS (1 << 24)   /* rows of a table */
#define BP_MAX_IDS (1 << 26)      /* ids of one call */
#define BP_MAX_WIDTH 8192         /* units of a residual stream: 16 for each of the 512 threads that keep a row's weights */
#define BP_MAX_TENSORS 65535      /* changes that are clipped together */

/* A table of n_tokens rows of `width` units, for up to max_ids ids a call.
 * 1 <= n_tokens <= BP_MAX_TOKENS, 1 <= max_ids <= BP_MAX_IDS.
 * Errors: BP_EINVAL, BP_ESHAPE (a BP_BF16 width that is no multiple of 8), BP_ENOMEM, BP_ECUDA. */
bp_status bp_embedding_create(int n_tokens, int width, int dtype, int max_ids, bp_embedding** out);
void bp_embedding_destroy(bp_embedding* layer);   /* NULL-safe; synchronises the device */

/* d_Y [n, width]: row i is scale * d_table[d_ids[i]], d_table [n_tokens, width].  An id of -1 is an empty
 * place: its row is zeros.  Any other id outside [0, n_tokens) gets zeros too, and is latched
 * for bp_embedding_check (BP_ESTATE).  A pattern of several tokens is a row of n * width units.  d_Y must
 * not overlap d_table.  Errors: BP_EINVAL (also a scale that is not finite), BP_ECUDA. */
bp_status bp_embed(bp_embedding* layer, const void* d_table, const int* d_ids, int n, float scale, void* d_Y,
                   void* stream);

/* d_G [n_tokens, width] = scale * the sum over the i with d_ids[i] = t of row i of d_D [n, width], for each
 * token t; zeros for a token without ids.  Ids that bp_embed gives zeros for have no part.  accumulate != 0
 * adds to d_G, and leaves rows of tokens without ids alone.  Rows of a token are added up in ascending i in pieces of at most
 * 32, and the pieces in few steps, so that the error does not grow with a token's rows (2^-24 of the magnitudes for each of
 * at most 190 additions in a row); where pieces begin depends on the other ids of the call.  Errors: as bp_embed. */
bp_status bp_embed_backward(bp_embedding* layer, const int* d_ids, int n, const void* d_D, float scale, float* d_G,
                            int accumulate, void* stream);

/* Wait for `stream`, then report and clear what the layer's kernels latched: BP_ESTATE (an id out of
 * range).  Errors: also BP_EINVAL, BP_ECUDA. */
bp_status bp_embedding_check(bp_embedding* layer, void* stream);

/* Norms of a row x of `width` values, with eps as the handle has it:
 *   BP_NORM_NONE   x itself;
 *   BP_NORM_RMS    w * x / sqrt(mean(x^2) + eps);
 *   BP_NORM_LAYER  w * (x - mean(x)) / sqrt(mean((x - mean(x))^2) + eps) + b. */
enum { BP_NORM_NONE = 0, BP_NORM_RMS = 1, BP_NORM_LAYER = 2 };

/* A stream of `width` units (at most BP_MAX_WIDTH) for up to max_rows rows and max_gates rows of gates a
 * call; norm_out: of a block's output, norm_in: before the next block; eps > 0 and finite.
 * Errors: BP_EINVAL, BP_ESHAPE (a BP_BF16 width that is no multiple of 8), BP_ENOMEM, BP_ECUDA. */
bp_status bp_residual_create(int width, int dtype, int max_rows, int max_gates, int norm_out, int norm_in, float eps,
                             bp_residual** out);
void bp_residual_destroy(bp_residual* stream);   /* NULL-safe; synchronises the device */

/* For each row t of the stream d_X [n, width] and of a block's output d_F [n, width]:
 *   d_Y = x + scale * gate * norm_out(f; d_wo, d_bo),
 *   d_H = norm_in(y; d_wi, d_bi), of y as it is stored.
 * d_F NULL: there is no block before; d_H is of x, and d_Y, where given, a copy of it (d_wo, d_bo and d_gate
 * are not read).  d_H NULL: the sum alone; BP_NORM_NONE takes no d_H.  d_Y may be NULL with d_F NULL only.
 * d_wo, d_wi [width]: NULL is 1; d_bo, d_bi [width], BP_NORM_LAYER only: NULL is 0.
 * d_gate [n_gates, width] or NULL (1; n_gates 0): row t has the gates g with d_offsets[g] <= t <
 * d_offsets[g + 1], d_offsets [n_gates + 1] on the device, from 0 to n; d_offsets NULL: one row of gates,
 * for all.  Rows outside every range have gates of 0 and nothing of f, whatever lies there (a NaN too): their y is x, their d_dF is
 * zeros, and they have no part in d_Gwo, d_Gbo and d_Ggate.  Offsets that do not ascend or leave [0, n] are
 * latched for bp_residual_check (results then mean nothing, and stay inside their buffers).
 * d_stats [n, 4] or NULL: mean and 1 / sqrt(...) of f, then of y, for the backward pass (0 and 1 where there
 * is no such norm; the mean is 0 for BP_NORM_RMS).
 * d_Y may be d_X, and d_H may be d_F; buffers must not overlap otherwise.
 * Errors: BP_EINVAL, BP_ECUDA; bp_residual_check. */
bp_status bp_residual_forward(bp_residual* stream_layer, const void* d_X, const void* d_F, int n, const float* d_wo,
                              const float* d_bo, const float* d_gate, const int* d_offsets, int n_gates, float scale,
                              const float* d_wi, const float* d_bi, void* d_Y, void* d_H, float* d_stats, void* stream);

/* The gradients for d_dY [n, width], that of y from what reads the stream later (NULL: 0), and d_dH [n, width],
 * that of h (NULL: 0); d_Y, d_F and d_stats as the forward call had and wrote them (d_Y is read if d_dH is
 * given; without a block before it is x).  With g = d_dY + that of y by way of h:
 *   d_dX [n, width]   g;
 *   d_dF [n, width]   that of f by way of scale * gate * g (needs d_F);
 *   d_Gwo, d_Gbo, d_Gwi, d_Gbi [width], d_Ggate [n_gates, width]: of weights, biases and gates, summed over
 *                     their rows.  Any of these seven may be NULL; one whose operand the handle's norms do not
 *                     have must be.
 * accumulate != 0 adds to the five sums instead of writing them.  d_dX may be d_dY, and d_dF may be d_dH; buffers
 * must not overlap otherwise.  Errors: as bp_residual_forward. */
bp_status bp_residual_backward(bp_residual* stream_layer, const void* d_Y, const void* d_F, int n, const float* d_wo,
                               const float* d_bo, const float* d_gate, const int* d_offsets, int n_gates, float scale,
                               const float* d_wi, const float* d_stats, const void* d_dY, const void* d_dH, void* d_dX,
                               void* d_dF, float* d_Gwo, float* d_Gbo, float* d_Ggate, float* d_Gwi, float* d_Gbi,
                               int accumulate, void* stream);

bp_status bp_residual_check(bp_residual* stream_layer, void* stream);   /* as bp_embedding_check; offsets */

/* The changes that are clipped together: n tensors (1 .. BP_MAX_TENSORS) of h_sizes[i] values of type h_dtypes[i] at
 * device address h_in[i], which go, clipped, to h_out[i] (h_out NULL: in place).  The three or four arrays are
 * host arrays and not kept; the device addresses are, and stay valid while the handle is used.  A size may
 * be 0; sizes add up to 2^40 at most.  Tensors lie on their values' boundaries.  A tensor's output is its input or apart from
 * every input, and outputs are apart from one another (else BP_EINVAL).
 * Errors: BP_EINVAL, BP_ENOMEM, BP_ECUDA. */
bp_status bp_clip_create(const void* const* h_in, void* const* h_out, const int64_t* h_sizes, const int* h_dtypes,
                         int n, bp_clip** out);
void bp_clip_destroy(bp_clip* clip);   /* NULL-safe; synchronises the device */

/* d_norm [1] (float32; may be NULL) = sqrt of the sum of the squares of all values; where it is above max_norm
 * every value is multiplied by max_norm / norm on its way to its output, else the outputs are the inputs.
 * Squares and sums neither overflow nor vanish (32 values at a time are float32's,
 * scaled by a power of two where need be; beyond they are float64), nor does max_norm / norm.  The norm of finite values may lie
 * above float32's largest: *d_norm is then infinity, the values are clipped all the same, and nothing is latched.  A NaN or an
 * infinity among the values clips nothing, and is latched for bp_clip_check; *d_norm is then that NaN or infinity.
 * max_norm >= 0; infinity: the norm alone, outputs are not written.  Errors: BP_EINVAL, BP_ECUDA. */
bp_status bp_clip_run(bp_clip* clip, float max_norm, float* d_norm, void* stream);

/* Wait for `stream`, then report and clear what was latched: BP_ENONFINITE.  Errors: also BP_EINVAL, BP_ECUDA. */
bp_status bp_clip_check(bp_clip* clip, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* BP_BLOCKS_H */
