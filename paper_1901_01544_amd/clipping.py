"""Clipping of the workers' gradients to a largest norm, in front of the compression step: binding of ``include/iwp_clip.h``.

    clipping.Tensors            which stretches of a flat buffer hold tensors, from the rows that ``iwp.Plan`` takes
    clipping.clip               norms of the workers' gradients over all tensors; the gradients scaled and clipped

Conventions are those of ``iwp``: outputs and workspace are the caller's, the call only enqueues kernels on ``stream`` and can be captured
into a graph.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import torch

from . import iwp


class Tensors:
    """Owner of an ``iwp_tensors``.  rows: (offset, elements, ...) per tensor, ascending; what follows in a row is not used."""

    def __init__(self, rows):
        rows = [(int(row[0]), int(row[1])) for row in rows]
        tab = (iwp.Layer * max(1, len(rows)))()
        for t, (offset, n) in zip(tab, rows):
            t.fill(offset, n)
        handle = C.c_void_p()
        iwp._check(iwp.load().iwp_tensors_create(tab, len(rows), C.byref(handle)), "iwp_tensors_create")
        self._h, self._address = handle, handle.value
        self.end = max(offset + n for offset, n in rows)

    def workspace_bytes(self, W: int) -> int:
        n = int(iwp.load().iwp_tensors_workspace_bytes(self._h, W))
        if n == 0:
            raise ValueError("1 to %d workers are wanted, not %d" % (iwp.IWP_MAX_WORKERS, W))
        return n

    def close(self):
        if getattr(self, "_h", None):
            iwp.load().iwp_tensors_destroy(self._h)
            self._h = self._address = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


_F32 = torch.float32


def _flat(buffers, what: str, end: int):
    for t in buffers:
        if t is not None and (t.dtype is not _F32 or t.numel() < end):
            raise ValueError("%s: flat float32 buffers of at least %d elements are wanted, not %s of %s" % (what, end, t.dtype, tuple(t.shape)))


def clip(tensors: Tensors, g: Sequence, out: Optional[Sequence], norm, workspace, max_norm: float = float("inf"), scale: float = 1.0,
         stream=None):
    """norm[p] = |scale| * norm of g[p] over all tensors; out[p] = g[p] * (scale * min(1, max_norm / norm[p])).

    g: one flat buffer a worker, None for a worker without a gradient.  out: likewise, out[p] may be g[p]; None: norms alone.  norm: [W].  max_norm: inf
    scales alone, with an infinite norm too.
    workspace: ``tensors.workspace_bytes(W)`` bytes."""
    W = len(g)
    out = [None] * W if out is None else out
    if len(out) != W:
        raise ValueError("out: %d buffers are wanted, not %d" % (W, len(out)))
    if norm.dtype is not _F32 or norm.shape != (W,):
        raise ValueError("norm: float32 of shape %s is wanted, not %s of %s" % ((W,), norm.dtype, tuple(norm.shape)))
    _flat(g, "g", tensors.end)
    if out is not g:
        _flat(out, "out", tensors.end)
    iwp._check(iwp._hot().iwp_clip(tensors._address, g, out, W, scale, max_norm, norm, workspace, iwp._bytes(workspace), iwp._stream(stream)),
               "clip")
