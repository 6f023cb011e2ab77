/*
 * iwp_clip.h -- C ABI of the clipping of the workers' gradients to a largest norm, in front of the
 * compression step of iwp.h.
 *
 * Conventions are those of iwp.h.
 */
#ifndef IWP_CLIP_H
#define IWP_CLIP_H

#include <stddef.h>
#include <stdint.h>

#include "iwp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The tensors of a flat buffer: which stretches of it hold elements.  Made from a layer table like a plan's, whose k and out_offset are
 * not used; what lies between the rows is neither read nor written.  Creating and destroying it are set-up calls like a plan's:
 * they allocate / free a device table (16 bytes per 2048 elements) on the current device and synchronise. */
typedef struct iwp_tensors iwp_tensors;

/* rows: host array, in ascending order without overlap, offset + n <= IWP_MAX_FLAT. */
int iwp_tensors_create(const iwp_layer* rows, uint32_t n_rows, iwp_tensors** tensors_out);
void iwp_tensors_destroy(iwp_tensors* tensors);
/* Workspace of iwp_clip for W workers; 0 without a handle or for W out of range.  256-byte aligned. */
size_t iwp_tensors_workspace_bytes(const iwp_tensors* tensors, uint32_t W);

/* Every worker's gradient times `scale` (of a loss that was scaled up, say: its inverse) and clipped to max_norm by its own norm over
 * all tensors:
 *   norm[p]   = |scale| * sqrt(sum of g[p][i]^2 over all tensors)
 *   out[p][i] = g[p][i] * (scale * min(1, max_norm / norm[p]))
 * The squares and their sum are binary64 (no gradient over- or underflows them), and so is the product, which is rounded once; norm is
 * rounded to binary32 (infinite where it lies above).  A norm of 0 leaves 0; a NaN among the gradients makes the norm and all of out NaN; an
 * infinity makes the norm infinite, what is infinite NaN and everything else 0, unless max_norm is INFINITY too: then nothing is clipped, the infinity
 * stays one and everything else is scaled.  So norm tells whether the step is to be taken.
 * g: host array of W device pointers to flat buffers, NULL for a worker without a gradient (norm 0, nothing written).  out: host array
 * of W device pointers, out[p] may be g[p] (then a gradient that stays as it is is not written), NULL there or as a whole: the norm alone.  norm:
 * device array of W binary32.  max_norm: INFINITY to scale alone.
 * IWP_EINVAL: pointers missing, W out of range, scale not finite, max_norm negative or NaN, an out[p] that overlaps another out or a g other
 * than g[p] itself; IWP_EALIGN: a buffer not 4-byte aligned, or the workspace. */
int iwp_clip(const iwp_tensors* tensors, const float* const* g, float* const* out, uint32_t W, double scale, double max_norm,
             float* norm, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* IWP_CLIP_H */
