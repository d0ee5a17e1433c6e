/*
 * libsoap's layer operators: the parts of a training step beside the optimizer's that its
 * matrices' gradients pass through, as stand-alone calls in the same library (include/soap.h).
 *
 *   layer_norm_*   layer normalisation of rows, and its backward pass with the weight's and
 *                  the bias's gradients
 *   layer_route_*  a mixture-of-experts router's decision: softmax, the k largest logits with
 *                  their gates, per-expert counts, the balance loss, and the logits' gradient
 *   layer_ffn_*    a gated feed-forward block, dense or over groups of rows with weights of their
 *                  own (a router's experts), and its backward pass
 *   layer_qk_*     norms of queries and keys for each head and their rotation by position, and the
 *                  backward pass
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

/* A matrix for each group: element (i, j) of group g at g * stride + i * ld + j, or, `columns`
 * nonzero, at g * stride + i + j * ld (column-major). */
typedef struct {
  void* data;
  int64_t ld, stride;
  int32_t columns;
} layer_matrix_t;

typedef enum { LAYER_SILU = 0, LAYER_GELU = 1 } layer_act_t;

/* A gated feed-forward block of `rows` rows x [hidden], for each group of rows with weights of its own:
 *   g = x Wg,  u = x Wu,  h = act(g) u,  y = h Wd
 *   silu(g) = g / (1 + e^-g),  gelu(g) = g Phi(g) (Phi: the normal distribution)
 * Wg, Wu: hidden x width, both row-major or both column-major; Wd: width x hidden; all of x's `type`.
 * offsets: device int32 [groups + 1]; rows offsets[g] .. offsets[g + 1] - 1 are group g's (none: an empty group).
 * Rows before offsets[0] and from offsets[groups] on are no group's: their y is 0 whatever they hold. NULL: groups
 * is 1 and every row its own. Offsets that fall, or are outside 0 .. rows, are raised to the largest before them and
 * cut at rows, and SOAP_STATUS_RANGE is ORed into *status.
 * pre: layer_ffn_pre_elems fp32 elements, 16-byte aligned, receives g and u for the backward pass (in an order of the
 * library's own), or NULL. Products are summed in fp32, g and u are fp32.
 * 16-bit types: h is rounded to the type before the second product, the backward pass's dg, du and h too, so that results
 * have two roundings, 1.4 of one in root mean square. fp16: what is above 65504 is then infinite, below 2^-14 it loses
 * bits, below 2^-25 it is 0 (dy may have to be scaled). Where rows * hidden <= 16384 and groups * hidden * width <= 2^23,
 * h, dg and du keep twice the type's bits and results have their own rounding alone: how exact a row is, and its last
 * bits, depend on the rows that share its call.
 * Infinite elements give the infinities and NaN of products in the type, with two exceptions that give NaN in a sum
 * that an infinity would decide: fp32 beside elements below 2^-62, which are used in parts that may be 0, and 16-bit
 * types where h, dg and du have twice the bits.
 * x, y: row i at element i * ld; y must not overlap an operand. status: NULL, or a device int32 (not cleared); where a
 * bounded wait gave up (soap_wait_limit), SOAP_STATUS_TIMEOUT is ORed into it and all results, pre among them, are NaN.
 * 0 <= rows <= 2^31 - 2^16; 1 <= hidden, width <= 65536; 1 <= groups <= 1024. `workspace`: 256-byte aligned,
 * layer_ffn_workspace_bytes bytes (0 for invalid sizes); aligned: nonzero if every matrix operand of the call
 * begins on a 16-byte boundary, with leading dimension and stride of whole 16-byte units (others are
 * copied to the workspace first). */
size_t layer_ffn_pre_elems(int64_t rows, int64_t width, int32_t groups);
size_t layer_ffn_workspace_bytes(int64_t rows, int64_t hidden, int64_t width, int32_t groups, int32_t type,
                                 int32_t aligned, int32_t backward);
soap_status_t layer_ffn_forward(int64_t rows, int64_t hidden, int64_t width, int32_t groups,
                                const int32_t* offsets, const void* x, int64_t ld_x, int32_t type,
                                const layer_matrix_t* gate, const layer_matrix_t* up, const layer_matrix_t* down,
                                int32_t act, void* y, int64_t ld_y, float* pre, int32_t* status, void* workspace,
                                size_t workspace_bytes, soap_stream_t stream);

/* The backward pass, from the forward call's pre:
 *   dh = dy Wd^T,  dg = dh u act'(g),  du = dh act(g)
 *   dx = dg Wg^T + du Wu^T,  dWg = x^T dg,  dWu = x^T du,  dWd = h^T dy
 * d_gate, d_up, d_down: receive the weights' gradients (`type`; 0 for an empty group; each in its weight's order:
 * columns as there), all three NULL: not formed. Rows of no group have dx 0, whatever their x and dy hold. Results
 * must not overlap an operand. */
soap_status_t layer_ffn_backward(int64_t rows, int64_t hidden, int64_t width, int32_t groups,
                                 const int32_t* offsets, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x,
                                 int32_t type, const layer_matrix_t* gate, const layer_matrix_t* up,
                                 const layer_matrix_t* down, int32_t act, const float* pre, void* dx, int64_t ld_dx,
                                 const layer_matrix_t* d_gate, const layer_matrix_t* d_up,
                                 const layer_matrix_t* d_down, int32_t* status, void* workspace,
                                 size_t workspace_bytes, soap_stream_t stream);

/* Heads of `dim` contiguous elements: of token s of sequence b, head h, at
 * b * batch_stride + s * token_stride + h * head_stride. */
typedef struct {
  void* data;
  int64_t batch_stride, token_stride, head_stride;
} layer_heads_t;

/* Queries and keys, `heads` and `kv_heads` of each of batch * length tokens: a root-mean-square norm for each
 * head and the rotation of its first `rotary` elements by the token's position:
 *   n = x / sqrt(mean(x^2) + eps),  m = n * weight  (the sum of x^2 is fp32: |x| up to 2^59),
 *   (a, b) -> (a c - b s, b c + a s) for the pairs (m_j, m_{j + rotary / 2}) or, `interleaved`,
 *   (m_2j, m_{2j + 1}), with c = cos[p][j], s = sin[p][j]; the other elements stay m
 * cos, sin: fp32 [places][rotary / 2], places < 2^31. positions: device int32, or int64 with positions_64, [batch * length],
 * or NULL: a token's place in its sequence. A position outside 0 .. places - 1 makes its token's results NaN, and
 * SOAP_STATUS_RANGE is ORed into *status (if not NULL; not cleared). q, k and the results: `type`;
 * q_weight, k_weight: dim elements of w_type (SOAP_F32 or `type`), either may be NULL (1). Results may be
 * the operands themselves (in place). Sums are fp32, each result is rounded once.
 * dim: even, 2 .. 512; rotary: even, 0 .. dim (0: cos, sin may be NULL, positions are not read);
 * heads, kv_heads: 0 .. 32768 (0: q, k and their results are not read and may be NULL); batch * length <=
 * 2^31 - 2^16; eps >= 0. Operands' strides may be 0 (one head or token for several); results' heads must not
 * overlap, nor a result's any operand's but its own. Heads whose parts are 16-byte aligned (strides,
 * rotary / 2 and dim / 2 of whole 16-byte units) move fastest. */
soap_status_t layer_qk_forward(int64_t batch, int64_t length, int32_t heads, int32_t kv_heads, int32_t dim,
                               int32_t rotary, int32_t interleaved, const layer_heads_t* q, const layer_heads_t* k,
                               int32_t type, const void* q_weight, const void* k_weight, int32_t w_type, float eps,
                               const float* cos, const float* sin, int64_t places, const void* positions,
                               int32_t positions_64, const layer_heads_t* q_out, const layer_heads_t* k_out,
                               int32_t* status, soap_stream_t stream);

/* The backward pass from the operands of the forward call: with dm the gradient turned back, g = dm * weight,
 *   dx = (g - n mean(g n)) / sqrt(mean(x^2) + eps),  dweight = sum over tokens and heads of dm n
 * dq, dk: the results' gradients; dx_q, dx_k: receive the operands' (may be dq, dk, q or k). d_qweight, d_kweight:
 * fp32 [dim] or both NULL (not formed); NaN where a position is out of range. `workspace`: 16-byte
 * aligned, layer_qk_workspace_bytes(...) bytes (NULL when neither is formed). */
size_t layer_qk_workspace_bytes(int64_t batch, int64_t length, int32_t heads, int32_t kv_heads, int32_t dim);
soap_status_t layer_qk_backward(int64_t batch, int64_t length, int32_t heads, int32_t kv_heads, int32_t dim,
                                int32_t rotary, int32_t interleaved, const layer_heads_t* dq,
                                const layer_heads_t* dk, const layer_heads_t* q, const layer_heads_t* k,
                                int32_t type, const void* q_weight, const void* k_weight, int32_t w_type, float eps,
                                const float* cos, const float* sin, int64_t places, const void* positions,
                                int32_t positions_64, const layer_heads_t* dx_q, const layer_heads_t* dx_k,
                                float* d_qweight, float* d_kweight, int32_t* status, void* workspace,
                                size_t workspace_bytes, soap_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* LAYER_H_ */
