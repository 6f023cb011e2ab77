/*
 * iwp_losses.h -- C ABI of the losses whose gradients the compression step of iwp.h takes:
 * softmax cross entropy and distillation through a language model's head, and the load balance
 * of a mixture of experts, each with its gradient.
 *
 * Conventions are those of iwp.h: device pointers, caller-owned buffers, kernels enqueued on
 * `hip_stream` and nothing else (no allocation, no synchronisation, no state between calls; a
 * HIP graph may capture them), argument errors found before anything is launched, the same bytes
 * for the same inputs.  What differs: rows may be strided (ld = elements from row to row, the
 * elements of a row lie together), and three types of data are taken:
 *   IWP_F32   products of binary32 operands as three products of their halves, sums in binary32: 22 bits
 *             of an element that is at least 2^-27 of its matrix's largest finite one (in h: of the
 *             tokens that count), 2^-49 of that one below; the logits' gradient likewise, against its
 *             token's coefficients; everything else in binary32
 *   IWP_BF16, IWP_F16   products of the operands as they are, sums in binary32; the logits'
 *             gradient is rounded to the operands' type before the two products that use it.
 *             IWP_BF16: the logits of the vocabulary's last piece (all of it, if it is worked through
 *             at once) are kept for the gradient in 16 bits, off by at most 2^-13 (1 + d) where d is the
 *             distance to the largest of 32 to 128 neighbouring entries' logits; those of the
 *             other pieces are computed again, in binary32
 * Softmax statistics, losses and sums are binary32 throughout.
 */
#ifndef IWP_LOSSES_H
#define IWP_LOSSES_H

#include <stddef.h>
#include <stdint.h>

#include "iwp.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { IWP_F32 = 0, IWP_BF16 = 1, IWP_F16 = 2 } iwp_dtype;

#define IWP_MAX_TOKENS (1u << 20)
#define IWP_MAX_DIM (1u << 16)
#define IWP_MAX_VOCAB (1u << 22)
#define IWP_MAX_TOP 1024u
#define IWP_MAX_HELD ((uint64_t)1 << 38)        /* tokens x vocabulary entries whose logits are held at a time */
#define IWP_MAX_EXPERTS 1024u

/* ------------------------------------------------------------------ the head */

/* Workspace of the two head calls.  tokens, dim, vocab: sizes; ld_w, w: the weight's rows as they will
 * be handed over (a weight of 16 bits whose rows are not 16-byte aligned is copied into the workspace
 * first, one of 32 bits is split there); top: the teacher's entries per token (0: cross entropy);
 * piece: vocabulary entries whose logits are held at a time (rounded up to 256), 0 = all of them.  The rest of the vocabulary is worked
 * through in pieces, whose logits are computed a second time for the gradient: at piece >= vocab nothing is
 * computed twice, below it the workspace holds a piece's logits instead of all of them (and 8 bytes, with a
 * teacher 12, per token and 32 to 128 entries of the vocabulary).  256-byte aligned.  0 for sizes that the calls refuse. */
size_t iwp_head_workspace_bytes(uint32_t tokens, uint32_t dim, uint32_t vocab, uint32_t dtype, const void* w, int64_t ld_w,
                                uint32_t top, uint32_t piece);

/* Softmax cross entropy of the head's logits z = h w^T (never stored as a whole), and its gradient.
 * h: [tokens, dim], w: [vocab, dim], of one type.  Token i counts if 0 <= target[i] < vocab and its
 * weight[i] (NULL: 1) is not 0; then
 *   loss[i] = weight[i] * (log sum_j exp z_ij - z_i,target[i])
 *   dh, dw  = gradients of scale * sum_i loss[i]
 * A token that does not count has loss 0, a dh row of zeros, and no part in dw whatever its row of h holds.  (A NaN or an
 * infinity in the row of a token that counts, in w or in a weight makes what depends on it NaN or infinite, as by the definition: a weight
 * its own token's loss and dh row, and dw; an infinity in w all losses and gradients, also where its logits are -inf.)  A token's dh
 * row has the same relative error whatever the weights are.  In dw a token's part is exact to that error or, where that is more,
 * to 2^-48 (IWP_F32) or 2^-37 (IWP_F16) of the largest coefficient (the weight times what it multiplies) times the largest |h|.
 * loss: [tokens], binary32.  dh: [tokens, dim], h's type, or NULL.  dw: [vocab, dim], of dw_dtype (the operands' type, or
 * IWP_F32 as the flat gradients of iwp.h are), or NULL.  Both gradients are written, not added to.
 * IWP_EINVAL: sizes of 0 (tokens may be 0) or above the limits, pointers missing, scale not finite, rows that overlap;
 * IWP_EALIGN: a buffer not aligned to its elements, or the workspace; IWP_ERANGE: ld of 2^23 or more. */
int iwp_head_cross_entropy(const void* h, int64_t ld_h, const void* w, int64_t ld_w, uint32_t tokens, uint32_t dim,
                           uint32_t vocab, uint32_t dtype, const int32_t* target, const float* weight, float scale,
                           uint32_t piece, float* loss, void* dh, int64_t ld_dh, void* dw, int64_t ld_dw, uint32_t dw_dtype,
                           void* workspace, size_t workspace_bytes, void* hip_stream);

/* Distillation from a teacher's top logits through the same head, mixed with the cross entropy of a label.
 * top_index, top_logit: [tokens, top], packed; entries with an index outside [0, vocab) or a logit of -inf are left out, an
 * index that occurs twice counts with the sum of its entries.  With q = softmax(top_logit / temperature) over the token's entries,
 * p the head's softmax at that temperature over the whole vocabulary, and t = temperature:
 *   loss[i] = weight[i] * (hard * CE_i + soft * t^2 * sum_k q_k (log q_k - log p_k))
 * The label's part is 0 where target[i] is outside [0, vocab) (or target is NULL), the teacher's where no entry is left; a token with
 * neither does not count.  Everything else as above. */
int iwp_head_distill(const void* h, int64_t ld_h, const void* w, int64_t ld_w, uint32_t tokens, uint32_t dim, uint32_t vocab,
                     uint32_t dtype, const int32_t* top_index, const float* top_logit, uint32_t top, float temperature,
                     float soft, const int32_t* target, float hard, const float* weight, float scale, uint32_t piece,
                     float* loss, void* dh, int64_t ld_dh, void* dw, int64_t ld_dw, uint32_t dw_dtype, void* workspace,
                     size_t workspace_bytes, void* hip_stream);

/* ------------------------------------------------------------------ the router */

size_t iwp_balance_workspace_bytes(uint32_t tokens, uint32_t experts);

/* Load balance of a router's choice.  x: [tokens, experts] logits; chosen: [tokens, slots] experts, packed, entries
 * outside [0, experts) are slots given to nobody; keep: [tokens] bytes, 0 = the token does not count, NULL = no token is left out by it.
 * A token whose logits are all -inf does not count either.
 * With N tokens that count, p = softmax(x), L = log sum exp x, share_e = counts[e] / (N * slots):
 *   counts[e] = slots given to expert e
 *   loss[0] = experts * sum_e share_e * mean(p_e),  loss[1] = mean(L^2)
 *   dx = gradient of balance * loss[0] + z * loss[1] (the shares are constants), zeros for tokens that do not count
 * N = 0: everything is 0.  loss: 2 binary32; counts: [experts] int32; dx: x's type, or NULL.  experts at most IWP_MAX_EXPERTS,
 * slots at most experts. */
int iwp_balance(const void* x, int64_t ld_x, uint32_t tokens, uint32_t experts, uint32_t dtype, const int32_t* chosen,
                uint32_t slots, const uint8_t* keep, float balance, float z, float* loss, int32_t* counts, void* dx,
                int64_t ld_dx, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* IWP_LOSSES_H */
