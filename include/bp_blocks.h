/*
 * bp_blocks.h -- C ABI of libbp.so, third part: what stands around the layers of
 * bp_experts.h in a model of blocks.
 *
 *   Embedding  rows of a table by token, and the pooled change of every token's row
 *              (a layer whose input is one unit out of many).
 *
 * The conventions of bp.h and bp_experts.h hold (row-major contiguous buffers, caller-owned device
 * memory, streams, status codes, bp_last_error; values float32 or bfloat16 as the handle's dtype says;
 * gates, norms' weights, biases, statistics and every change G float32 in both; BP_BF16 rows are
 * multiples of 8 units on 16-byte boundaries, float32 and int buffers lie on 4-byte boundaries).  Values
 * are computed and summed in float32 and rounded once, on the way out.  Besides:
 *   - A handle belongs to the device that was current when it was made; calls with another
 *     one current are refused (BP_EINVAL).
 *   - Handles own scratch that each call reuses: calls on one handle, and graphs captured from
 *     them, belong on one stream at a time.  Compute calls allocate nothing and may be captured.
 *   - Results do not depend on the launch: every sum has one order for given sizes.
 */
#ifndef BP_BLOCKS_H
#define BP_BLOCKS_H

#include "bp.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct bp_embedding bp_embedding;

#define BP_MAX_TOKENS (1 << 24)   /* rows of a table */
#define BP_MAX_IDS (1 << 26)      /* ids of one call */

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
 * adds to d_G, and leaves rows of tokens without ids alone.  Rows of a token are added in
 * ascending i, 32 at a time.  Errors: as bp_embed. */
bp_status bp_embed_backward(bp_embedding* layer, const int* d_ids, int n, const void* d_D, float scale, float* d_G,
                            int accumulate, void* stream);

/* Wait for `stream`, then report and clear what the layer's kernels latched: BP_ESTATE (an id out of
 * range).  Errors: also BP_EINVAL, BP_ECUDA. */
bp_status bp_embedding_check(bp_embedding* layer, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* BP_BLOCKS_H */
