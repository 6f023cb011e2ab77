/*
 * iwp_experts.h -- C ABI of a routed layer's operators: the choice of experts with its gradient, and the
 * products of every token's rows with the matrices of the experts chosen for it, with theirs.
 *
 * Conventions are those of iwp_losses.h: device pointers, caller-owned buffers, kernels enqueued on
 * `hip_stream` and nothing else, argument errors found before anything is launched, the same bytes
 * for the same inputs, strided rows (ld = elements from row to row), data of iwp_dtype.
 */
#ifndef IWP_EXPERTS_H
#define IWP_EXPERTS_H

#include <stddef.h>
#include <stdint.h>

#include "iwp_losses.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { IWP_SOFTMAX = 0, IWP_SIGMOID = 1 } iwp_scores;

#define IWP_MAX_ROWS (1u << 24)                 /* tokens x slots of the products */

/* ------------------------------------------------------------------ the choice */

/* Chooses `slots` experts for every token from a router's logits.  x: [tokens, experts]; with s = softmax(x) over
 * the token's experts or 1 / (1 + exp(-x)), and bias: [experts] binary32, or NULL:
 *   c_e        by which experts are chosen: s_e + bias_e in binary64, without a bias the logit x_e, in whose order the scores are
 *                (also where binary64 does not tell them apart)
 *   groups     the experts in `groups` equal runs, of which a token may use the top_groups with the largest sum of their
 *                group_top (1 or 2) largest c; without a bias two of a group are added as scores, in binary64
 *   chosen[k]  the experts with the largest c there, the largest first; among equals (of experts and of groups) the lower index
 *   weight[k]  scale * s_e of the k-th, with `renormalise` scale * s_e / (sum of s over the token's chosen experts); the bias has no part in it
 * Experts whose logit is -inf or NaN or whose c is -inf or NaN are never chosen; slots that are left over hold -1 and weight 0, and
 * so do all slots of tokens with keep[i] == 0 (keep: [tokens] bytes, NULL = every token counts).  A token with a NaN among its logits has
 * weights of NaN.  A logit of +inf makes a softmax NaN, as by the definition; such a token's weights are NaN, its choice without a bias is
 * by the logits' order, but where groups go by two scores there is none.
 * chosen: [tokens, slots] int32, weight: [tokens, slots] binary32, packed: `chosen` is what iwp_balance and
 * iwp_expert_product take.  No workspace.
 * IWP_EINVAL: experts of 0 or above IWP_MAX_EXPERTS, tokens above IWP_MAX_TOKENS (0 tokens: nothing is done), groups that do not divide the
 * experts, slots of 0 or more than top_groups * experts / groups, group_top above experts / groups, scale not finite, pointers missing,
 * ld_x < experts; IWP_EALIGN: a buffer not aligned to its elements. */
int iwp_route(const void* x, int64_t ld_x, uint32_t tokens, uint32_t experts, uint32_t dtype, const float* bias,
              uint32_t scores, uint32_t groups, uint32_t top_groups, uint32_t group_top, uint32_t renormalise, float scale,
              const uint8_t* keep, int32_t* chosen, float* weight, uint32_t slots, void* hip_stream);

/* The logits' gradient: dx = plus + sum_k dweight[k] * (gradient of weight[k]), rounded once.  chosen, dweight: [tokens, slots], packed,
 * chosen[] distinct experts as iwp_route wrote them; entries outside [0, experts) are left out, whatever their dweight.  plus: NULL, or
 * another gradient of x of its type (that of iwp_balance, say), which may be dx itself.  With D_j the dweight of the slot that holds j, or 0:
 *   softmax                dx_j = scale s_j (D_j - sum_k dweight_k s_k)
 *   softmax, renormalised  dx_j = scale v_j (D_j - sum_k dweight_k v_k) for chosen j, else 0; v = s / (sum of s over the chosen)
 *   sigmoid                dx_j = scale s_j (1 - s_j) D_j
 *   sigmoid, renormalised  dx_j = scale v_j (1 - s_j) (D_j - sum_k dweight_k v_k) for chosen j
 * Rows of tokens with keep[i] == 0 are plus, or 0.  An expert that occurs twice in a row of chosen[] counts as two slots.  Everything else as above. */
int iwp_route_gradient(const void* x, int64_t ld_x, uint32_t tokens, uint32_t experts, uint32_t dtype, const int32_t* chosen,
                       const float* dweight, uint32_t slots, uint32_t scores, uint32_t renormalise, float scale,
                       const uint8_t* keep, const void* plus, int64_t ld_plus, void* dx, int64_t ld_dx, void* hip_stream);

/* ------------------------------------------------------------------ the products */

/* Products of rows with the matrices of the experts chosen for them.  A row for every slot: row i * slots + k goes to expert chosen[i, k].
 *   x       [tokens, in], with every token's row for each of its slots, or with x_by_slot [tokens * slots, in], a row for each
 *   w       [experts, out, in]: ld_w elements from row to row, step_w from matrix to matrix
 *   chosen  [tokens, slots] int32, packed, as iwp_route writes it; entries outside [0, experts) are slots that nobody got
 *   y       [tokens * slots, out]: y_r = W_chosen[r] x_r, zeros for slots of nobody
 * All of one type, sums in binary32, rounded once.  Matrices of experts without rows are not read, except where w is copied (below), which takes all of
 * it.  An infinity or a NaN in a row, or in an expert's matrix, shows in what depends on it by the definition, where an infinity may also make NaN,
 * and nowhere else.
 * Workspace: iwp_expert_product_workspace_bytes with the same sizes, 256-byte aligned; it has room for the rows gathered by expert
 * and, where the rows of a w of 16 bits cannot be read by 16 bytes where they lie (address, ld_w, step_w and in), for a copy of w.
 * IWP_EINVAL: sizes of 0 (tokens may be 0) or above the limits (IWP_MAX_TOKENS, IWP_MAX_ROWS slots, IWP_MAX_EXPERTS, IWP_MAX_DIM for in and
 * out; rows times a width, and elements of all matrices, of some 2^36 and more, which no launch takes), slots above experts, pointers missing, rows that overlap (ld below the width; step below out rows); IWP_EALIGN: a
 * buffer not aligned to its elements, or the workspace; IWP_ERANGE: rows that lie 2^24 bytes or more apart. */
size_t iwp_expert_product_workspace_bytes(uint32_t tokens, uint32_t slots, uint32_t experts, uint32_t in, uint32_t out,
                                          uint32_t dtype, const void* w, int64_t ld_w, int64_t step_w, uint32_t x_by_slot,
                                          uint32_t gradient);
int iwp_expert_product(const void* x, int64_t ld_x, uint32_t x_by_slot, const void* w, int64_t ld_w, int64_t step_w,
                       uint32_t tokens, uint32_t slots, uint32_t experts, uint32_t in, uint32_t out, uint32_t dtype,
                       const int32_t* chosen, void* y, int64_t ld_y, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Its gradients.  dy: [tokens * slots, out], of x's type; rows of slots of nobody are not read.
 *   dx  like x, or NULL: W_chosen[r]^T dy_r of a slot's row (zeros for nobody's), or its sum over the token's slots, in binary32 and in their order
 *   dw  [experts, out, in], of dw_dtype (x's type, or IWP_F32 as the flat gradients of iwp.h are), or NULL: the sum over an expert's rows of
 *       dy_r x_r^T, zeros for an expert without rows
 * Both are written, not added to.  Workspace: with gradient = 1. */
int iwp_expert_product_gradient(const void* x, int64_t ld_x, uint32_t x_by_slot, const void* w, int64_t ld_w, int64_t step_w,
                                uint32_t tokens, uint32_t slots, uint32_t experts, uint32_t in, uint32_t out, uint32_t dtype,
                                const int32_t* chosen, const void* dy, int64_t ld_dy, void* dx, int64_t ld_dx, void* dw,
                                int64_t ld_dw, int64_t step_dw, uint32_t dw_dtype, void* workspace, size_t workspace_bytes,
                                void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* IWP_EXPERTS_H */
