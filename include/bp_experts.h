/*
 * bp_experts.h -- C ABI of libbp.so, second part: layers whose weights depend on
 * the pattern.
 *
 *   Router    chooses k of E experts for each pattern, their gates, and the order
 *             in which the experts' rows lie;
 *   Experts   E fully connected layers of one shape; each row is multiplied by the
 *             weights of its own expert (products grouped by expert, ragged);
 *   Mix       each pattern's gated sum of its experts' outputs;
 *   Adapters  one shared layer plus, for each request, the low-rank change of that
 *             request's adapter.
 *
 * Every one has its forward pass and its gradients.  The conventions of bp.h hold
 * (row-major contiguous buffers, caller-owned device memory, streams, status codes,
 * bp_last_error), and besides:
 *   - Values are float32 (BP_F32) or bfloat16 (BP_BF16) as the handle's or the call's
 *     dtype says; biases, gates, scales, U and every change G are float32 in both.
 *     Products are summed in float32 (or by the tensor cores in float32) and rounded
 *     once, on the way out.
 *   - BP_BF16 needs n_in and n_out to be multiples of 8 and pattern, weight, U and G
 *     buffers on 16-byte boundaries; float32 and int buffers otherwise lie on 4-byte
 *     boundaries.
 *   - A call may have no rows (n or n_rows 0); row buffers may then be NULL.  Rows (of a router and
 *     a mix: n * k, of adapters: max_rows * BP_MAX_RANK) and requests are at most INT_MAX - 1023.
 *   - Index buffers (source, offsets, adapter, place) lie on the device and are not
 *     read by the host.  Kernels clamp offsets to [0, n_rows] and to ascending order,
 *     read a source row outside [0, n_x) as row 0, and treat an adapter outside
 *     [0, n_adapters) other than -1 as none; each of these latches an error that the
 *     handle's check call reports as BP_ESTATE.  A place outside [0, n_rows) takes no
 *     part in a mix.
 *   - Handles own scratch that each call reuses: calls on one handle belong on one
 *     stream at a time.  Compute calls allocate nothing and may be captured.
 *   - Results do not depend on the launch: every sum has one order for given sizes.
 */
#ifndef BP_EXPERTS_H
#define BP_EXPERTS_H

#include "bp.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct bp_router bp_router;
typedef struct bp_experts bp_experts;
typedef struct bp_adapters bp_adapters;

#define BP_MAX_EXPERTS 512     /* experts of a router or of an expert layer */
#define BP_MAX_CHOICES 16      /* experts of one pattern (k) */
#define BP_MAX_RANK 128        /* rank of an adapter */

/* Gates of the chosen experts S of a pattern with logits z:
 *   BP_GATES_CHOSEN  g_j = exp(z_j) / sum over S of exp(z);
 *   BP_GATES_ALL     g_j = exp(z_j) / sum over all experts of exp(z). */
enum { BP_GATES_CHOSEN = 0, BP_GATES_ALL = 1 };

/* A router for up to max_patterns patterns a call; dtype: of the logits and their
 * gradient.  1 <= n_experts <= BP_MAX_EXPERTS, 1 <= k <= min(n_experts,
 * BP_MAX_CHOICES).  Errors: BP_EINVAL, BP_ENOMEM, BP_ECUDA. */
bp_status bp_router_create(int n_experts, int k, int dtype, int max_patterns, int gates,
                           bp_router** out);
void bp_router_destroy(bp_router* router);   /* NULL-safe; synchronises the device */

/* Choice, gates and order for n patterns with logits d_logits [n, E].
 *   d_expert [n, k]   the k experts of largest logit, largest first, ties to the lowest
 *                     index; -1 where fewer than k logits exceed -infinity (a closed
 *                     expert has the logit -infinity);
 *   d_gate [n, k]     their gates, 0 beside -1.  A pattern with a NaN logit has NaN
 *                     gates; NaN logits are not chosen;
 *   d_offsets [E + 1] the rows of expert e are [offsets[e], offsets[e + 1]), by
 *                     ascending pattern;
 *   d_source [n * k]  the pattern of each row, -1 from row offsets[E] on;
 *   d_place [n, k]    the row of each choice, -1 beside -1.
 * Errors: BP_EINVAL, BP_ECUDA. */
bp_status bp_route(bp_router* router, const void* d_logits, int n, int* d_expert, float* d_gate,
                   int* d_offsets, int* d_source, int* d_place, void* stream);

/* d_dlogits [n, E] (the router's dtype, written in full) from the gradient d_dgate [n, k]
 * of the gates; d_expert and d_gate as bp_route wrote them.  dgate beside an expert of -1
 * is not read.  Errors: BP_EINVAL, BP_ECUDA. */
bp_status bp_route_backward(bp_router* router, const void* d_logits, int n, const int* d_expert,
                            const float* d_gate, const float* d_dgate, void* d_dlogits, void* stream);

/* d_Y [n, n_out] = sum over j < k of d_gate[t, j] * d_H[d_place[t, j]], d_H [n_rows, n_out];
 * d_gate NULL: gates of 1 (the sum of a pattern's rows, as the gradient of inputs that
 * several experts read).  1 <= k <= BP_MAX_CHOICES; BP_BF16 needs n_out a multiple of 8.
 * No handle, no scratch.  Errors: BP_EINVAL, BP_ESHAPE, BP_ECUDA. */
bp_status bp_mix(const void* d_H, int n_rows, const int* d_place, const float* d_gate, int n, int k,
                 int n_out, int dtype, void* d_Y, void* stream);

/* The gradients of bp_mix for d_D [n, n_out], the gradient of Y:
 *   d_dH [n_rows, n_out]  row place[t, j] is gate[t, j] * D[t]; rows that no place names
 *                         are left alone;
 *   d_dgate [n, k]        D[t] . H[place[t, j]], 0 where place takes no part (may be NULL;
 *                         d_H is then not read and may be NULL).
 * Every row is named by one place at most.  Errors: as bp_mix. */
bp_status bp_mix_backward(const void* d_D, const void* d_H, int n_rows, const int* d_place,
                          const float* d_gate, int n, int k, int n_out, int dtype, void* d_dH,
                          float* d_dgate, void* stream);

/* E layers of n_in inputs and n_out units for up to max_rows rows a call.
 * Errors: BP_EINVAL, BP_ESHAPE (BP_BF16 sizes that are not multiples of 8), BP_ENOMEM,
 * BP_ECUDA. */
bp_status bp_experts_create(int n_experts, int n_in, int n_out, int dtype, int max_rows,
                            bp_experts** out);
void bp_experts_destroy(bp_experts* layer);   /* NULL-safe; synchronises the device */

/* Rows [offsets[e], offsets[e + 1]) of d_Y [n_rows, n_out] = W_e x + b_e, with squash != 0
 * the logistic of it.  d_W [E, n_out, n_in], d_b [E, n_out] or NULL.  Row r's input is
 * d_X[d_source[r]], d_X [n_x, n_in]; d_source NULL: d_X[r].  Rows in no group are left
 * alone.  d_Y must not overlap d_X.  Errors: BP_EINVAL, BP_ECUDA; bp_experts_check. */
bp_status bp_experts_forward(bp_experts* layer, const void* d_W, const float* d_b, const void* d_X,
                             int n_x, const int* d_source, const int* d_offsets, int n_rows,
                             int squash, void* d_Y, void* stream);

/* The gradients for d_D [n_rows, n_out], the gradient of W_e x + b_e (a delta of the
 * framework: the squashing function's slope is in it):
 *   d_dX [n_rows, n_in]    W_e^T d of each row in a group, in the rows' order (bp_mix with
 *                          gates of 1 adds up the rows of a pattern); squash != 0: times
 *                          x (1 - x), the hidden delta of an input that is itself a
 *                          logistic's output.  May be NULL; must not overlap d_X or d_D.
 *   d_GW [E, n_out, n_in]  sum over the expert's rows of d x^T, zeros for one without rows;
 *   d_Gb [E, n_out]        sum over the expert's rows of d.  Either may be NULL.
 * accumulate != 0 adds to d_GW and d_Gb instead of writing them.  d_W may be NULL without
 * d_dX.  Errors: BP_EINVAL, BP_ECUDA; bp_experts_check. */
bp_status bp_experts_backward(bp_experts* layer, const void* d_W, const void* d_X, int n_x,
                              const int* d_source, const int* d_offsets, int n_rows, const void* d_D,
                              int squash, void* d_dX, float* d_GW, float* d_Gb, int accumulate,
                              void* stream);

/* Wait for `stream`, then report and clear what the layer's kernels latched: BP_ETIMEOUT (a
 * bounded wait ran out), BP_ESTATE (an index out of range).  Errors: also BP_EINVAL, BP_ECUDA. */
bp_status bp_experts_check(bp_experts* layer, void* stream);

/* n_adapters adapters of rank `rank` (1 .. BP_MAX_RANK) beside one layer of n_in inputs and
 * n_out units, for calls of up to max_rows rows and max_requests requests.
 * Errors: as bp_experts_create. */
bp_status bp_adapters_create(int n_adapters, int rank, int n_in, int n_out, int dtype, int max_rows,
                             int max_requests, bp_adapters** out);
void bp_adapters_destroy(bp_adapters* layer);   /* NULL-safe; synchronises the device */

/* Request i has the rows [offsets[i], offsets[i + 1]) (offsets[0] = 0, offsets[n_requests] =
 * n_rows; a request may have none) and the adapter a = d_adapter[i], or none (-1):
 *   d_U [n_rows, rank]  = A_a x             (zeros without an adapter)
 *   d_Y [n_rows, n_out] = W x + b + scale_a B_a^T u, with squash != 0 the logistic of it.
 * d_W [n_out, n_in], d_b [n_out] or NULL, d_A [n_adapters, rank, n_in], d_B [n_adapters, rank,
 * n_out] (both by rank, so that their rows run along the layer's units), d_scale
 * [n_adapters] or NULL (1), d_X [n_rows, n_in].  d_U is kept for the backward pass.
 * Rows outside every request get the shared layer alone.
 * Errors: BP_EINVAL, BP_ECUDA; bp_adapters_check. */
bp_status bp_adapters_forward(bp_adapters* layer, const void* d_W, const float* d_b, const void* d_A,
                              const void* d_B, const float* d_scale, const void* d_X,
                              const int* d_offsets, const int* d_adapter, int n_requests, int n_rows,
                              int squash, float* d_U, void* d_Y, void* stream);

/* The gradients for d_D [n_rows, n_out], the gradient of the sum before the squashing function;
 * the shared layer has none (its weights are not trained here).  With v = scale_a B_a d:
 *   d_dX [n_rows, n_in]              W^T d + A_a^T v, squash != 0: times x (1 - x); may be NULL; must
 *                                    not overlap d_X or d_D;
 *   d_GA [n_adapters, rank, n_in]    sum over the rows of the adapter's requests of v x^T;
 *   d_GB [n_adapters, rank, n_out]   scale_a times the sum of u d^T.  Either may be NULL.
 * accumulate != 0 adds to d_GA and d_GB; else adapters without rows get zeros.
 * Errors: BP_EINVAL, BP_ECUDA; bp_adapters_check. */
bp_status bp_adapters_backward(bp_adapters* layer, const void* d_W, const void* d_A, const void* d_B,
                               const float* d_scale, const void* d_X, const float* d_U,
                               const int* d_offsets, const int* d_adapter, int n_requests, int n_rows,
                               const void* d_D, int squash, void* d_dX, float* d_GA, float* d_GB,
                               int accumulate, void* stream);

bp_status bp_adapters_check(bp_adapters* layer, void* stream);   /* as bp_experts_check */

#ifdef __cplusplus
}
#endif

#endif /* BP_EXPERTS_H */
