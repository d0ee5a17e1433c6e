/*
 * libsoap's layer operators: the parts of a training step beside the optimizer's that its
 * matrices' gradients pass through, as stand-alone calls in the same library (include/soap.h).
 *
 *   layer_norm_*   layer normalisation of rows, and its backward pass with the weight's and
 *                  the bias's gradients
 *   layer_route_*  a mixture-of-experts router's decision: softmax, the k largest logits with
 *                  their gates, per-expert counts, the balance loss, and the logits' gradient
 *
 * Conventions: those of include/soap.h (stream-ordered calls, host-side validation that returns
 * a status code before anything is enqueued, no kernel traps, the caller owns every buffer,
 * workspaces included) with these differences: a row-major operand may have any alignment its
 * type allows and any leading dimension >= its width (rows that are no whole 16-byte units may
 * take longer), and its type is one of soap_dtype_t. Sums, statistics and exponentials are fp32
 * whatever the type (e^x is the hardware's 2^(x log2 e), relative error 2^-22 + |x| 2^-24); every
 * result is rounded once. The calls run on the
 * device that is current for the calling thread, which must be the operands' and the stream's.
 * The results do not depend on scheduling: the same inputs give the same bits.
 */
#ifndef LAYER_H_
#define LAYER_H_

#include <stddef.h>
#include <stdint.h>

#include "soap.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Layer norm of `rows` rows of `width` elements:
 *   mu = mean(x), rstd = 1 / sqrt(mean((x - mu)^2) + eps), y = (x - mu) rstd * weight + bias
 * x, y: x_type, row i at element i * ld; y may be x (in place). weight, bias: `width` elements
 * of w_type (SOAP_F32 or x_type), either may be NULL (1, 0). mean, rstd: fp32 [rows] for the
 * backward pass, either may be NULL. status: NULL, or a device int32 into which the kernels OR
 * SOAP_STATUS_TIMEOUT if a bounded internal wait gave up (see soap_wait_limit; not cleared): the rows
 * concerned, forward also their statistics, and backward dweight and dbias are then NaN. rows = 0 does nothing.
 * SOAP_ERR_INVALID_ARG for rows < 0 or > 2^31 - 2^16, width < 1, a leading dimension below width, a
 * type out of range, a null or misaligned pointer, or eps < 0. */
soap_status_t layer_norm_forward(int64_t rows, int64_t width, const void* x, int64_t ld_x, int32_t x_type,
                                 const void* weight, const void* bias, int32_t w_type, float eps, void* y,
                                 int64_t ld_y, float* mean, float* rstd, int32_t* status,
                                 soap_stream_t stream);

/* The backward pass, from the forward pass's mean and rstd; with xh = (x - mu) rstd, g = dy * weight:
 *   dx = rstd (g - mean(g) - xh mean(g xh)),  dweight = sum over rows of dy xh,  dbias = sum of dy
 * dy, x, dx: x_type (dx may be dy or x). weight: as given forward (NULL: 1). dweight, dbias: fp32
 * [width] or NULL (not formed); rows = 0 sets them to 0. `workspace`: 16-byte aligned device
 * memory of layer_norm_workspace_bytes(rows, width) bytes for the per-CTA column sums (not needed,
 * and may be NULL, when neither gradient is formed). status: as forward. */
size_t layer_norm_workspace_bytes(int64_t rows, int64_t width);
soap_status_t layer_norm_backward(int64_t rows, int64_t width, const void* dy, int64_t ld_dy, const void* x,
                                  int64_t ld_x, int32_t x_type, const float* mean, const float* rstd,
                                  const void* weight, int32_t w_type, void* dx, int64_t ld_dx, float* dweight,
                                  float* dbias, void* workspace, size_t workspace_bytes, int32_t* status,
                                  soap_stream_t stream);

/* A router's decision for `tokens` rows z of `experts` logits (row i at element i * ld):
 *   p = softmax(z); chosen: the k largest logits, by value and then by the lower index
 *   gates = p of the chosen, divided by their sum if `normalize`
 *   counts_e = number of tokens that chose e, n = number of tokens counted
 *   loss = coef * experts / (k n) * sum_e counts_e * mean_probs_e,  mean_probs = sum of p / n
 * (loss = coef for a perfectly balanced choice).
 * mask: NULL, or one byte per token; a token whose byte is 0 is left out whatever its row holds:
 * indices -1, gates 0, no part in counts, n, mean_probs or the loss. An expert whose logit is -inf
 * is never chosen: a row with fewer than k finite logits has -1 and 0 in the remaining places, one
 * with none takes no part in mean_probs and is not counted in n. A row that is not masked and
 * holds a NaN or +inf chooses nothing, has NaN gates and makes mean_probs and the loss NaN, and
 * SOAP_STATUS_NONFINITE is ORed into *status (if not NULL; it is not cleared).
 * indices: int32 [tokens][k]; gates: fp32 [tokens][k]; counts: int32 [experts]; live: int32 [1],
 * receives n; mean_probs: fp32 [experts] or NULL; loss: fp32 [1]; stats: fp32 [tokens][2], 8-byte
 * aligned, for the backward pass (a row's largest logit and 1 / sum of e^(z - largest)), or NULL.
 * tokens = 0 gives zeros.
 * 1 <= experts <= 1024, 1 <= k <= min(experts, 32), 0 <= tokens < 2^31. `workspace`: 16-byte
 * aligned, layer_route_workspace_bytes(tokens, experts) bytes. */
size_t layer_route_workspace_bytes(int64_t tokens, int32_t experts);
soap_status_t layer_route_forward(int64_t tokens, int32_t experts, int32_t k, const void* logits, int64_t ld,
                                  int32_t type, const uint8_t* mask, int32_t normalize, float coef,
                                  int32_t* indices, float* gates, float* stats, int32_t* counts,
                                  int32_t* live, float* mean_probs, float* loss, int32_t* status,
                                  void* workspace, size_t workspace_bytes, soap_stream_t stream);

/* The logits' gradient from the gates' (fp32 [tokens][k], or NULL for zero) and the loss's (dloss), the
 * choice itself and the counts held constant:
 *   dp = coef dloss experts / (k n^2) * counts + (what reaches p through the gates),
 *   dz_e = p_e (dp_e - sum_j p_j dp_j)
 * dlogits: `type`, row i at element i * ld_d (may be logits when ld_d = ld). Rows that are masked or
 * not counted get zeros; a row with a NaN or +inf gets NaN. normalize, coef, mask, indices, stats,
 * counts, live: those of the forward call (indices may be NULL without dgates). */
soap_status_t layer_route_backward(int64_t tokens, int32_t experts, int32_t k, const void* logits, int64_t ld,
                                   int32_t type, const uint8_t* mask, int32_t normalize, float coef, float dloss,
                                   const int32_t* indices, const float* stats, const int32_t* counts,
                                   const int32_t* live, const float* dgates, void* dlogits, int64_t ld_d,
                                   soap_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* LAYER_H_ */
