"""Losses of a language model with the gradients that the compression step takes: binding of ``include/iwp_losses.h``.

    losses.head_cross_entropy   softmax cross entropy through the head, in pieces of the vocabulary
    losses.head_distill         distillation from a teacher's top logits through the head, mixed with the label
    losses.balance              load balance of a router's choice of experts, with the experts' counts

Outputs and workspaces are the caller's, as in ``iwp``: nothing is allocated, and the calls only enqueue kernels on ``stream``
(the current one if not given), so they can be captured into a graph.  Rows of matrices may be strided.  ``dw`` may be a
view into the flat binary32 gradients that ``iwp.step_segmented`` takes, whatever the operands' type is.  Refusals are
``ValueError`` for tensors that do not fit each other, ``iwp.IwpError`` for what the library turns away.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import iwp

F32, BF16, F16 = 0, 1, 2
_DTYPE = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


def _dtype(t, what: str) -> int:
    code = _DTYPE.get(t.dtype)
    if code is None:
        raise ValueError("%s: float32, bfloat16 or float16 is wanted, not %s" % (what, t.dtype))
    return code


def _matrix(t, what: str, rows: int, columns: int, dtype=None):
    """(address, elements from row to row) of a device matrix whose rows lie together."""
    if t.shape != (rows, columns):
        raise ValueError("%s: a matrix of %d x %d is wanted, not %s" % (what, rows, columns, tuple(t.shape)))
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s: %s is wanted, not %s" % (what, dtype, t.dtype))
    if not t.is_cuda:
        raise ValueError("%s: a device tensor is wanted" % what)
    ld, step = t.stride()
    if step != 1 and columns > 1:
        raise ValueError("%s: the elements of a row have to lie together" % what)
    return t.data_ptr(), max(ld, columns) if rows <= 1 else ld


def _packed(t, what: str, shape, dtype) -> Optional[int]:
    if t is None:
        return None
    if t.shape != shape or t.dtype != dtype:
        raise ValueError("%s: %s of shape %s is wanted, not %s of %s" % (what, dtype, shape, t.dtype, tuple(t.shape)))
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s: a contiguous device tensor is wanted" % what)
    return t.data_ptr()


def head_workspace_bytes(h, w, top: int = 0, piece: int = 0) -> int:
    """Workspace of the head calls on these tensors.  piece: vocabulary entries whose logits are held at a time (0: all)."""
    (tokens, dim), vocab = h.shape, w.shape[0]
    address, ld = _matrix(w, "w", vocab, dim, h.dtype)
    n = iwp.load().iwp_head_workspace_bytes(tokens, dim, vocab, _dtype(h, "h"), address, ld, top, piece)
    if n == 0:
        raise ValueError("sizes that the head calls refuse: %d tokens, %d wide, %d entries, %d of a teacher's"
                         % (tokens, dim, vocab, top))
    return int(n)


def _head(h, w, loss, dh, dw, weight, target):
    if h.dim() != 2 or w.dim() != 2:
        raise ValueError("h and w: matrices are wanted")
    (tokens, dim), vocab = h.shape, w.shape[0]
    code = _dtype(h, "h")
    h_at, ld_h = _matrix(h, "h", tokens, dim)
    w_at, ld_w = _matrix(w, "w", vocab, dim, h.dtype)
    dh_at, ld_dh = (None, 0) if dh is None else _matrix(dh, "dh", tokens, dim, h.dtype)
    dw_at, ld_dw = (None, 0) if dw is None else _matrix(dw, "dw", vocab, dim)
    dw_code = code if dw is None else _dtype(dw, "dw")
    if dw_code not in (code, F32):
        raise ValueError("dw: %s or float32 is wanted, not %s" % (h.dtype, dw.dtype))
    return ((h_at, ld_h, w_at, ld_w, tokens, dim, vocab, code), _packed(target, "target", (tokens,), torch.int32),
            _packed(weight, "weight", (tokens,), torch.float32),
            (_packed(loss, "loss", (tokens,), torch.float32), dh_at, ld_dh, dw_at, ld_dw, dw_code))


def head_cross_entropy(h, w, target, loss, dh, dw, workspace, weight=None, scale: float = 1.0, piece: int = 0, stream=None):
    """loss[i] = weight[i] * cross entropy of softmax(h[i] w^T) against target[i]; dh, dw = gradients of scale * loss.sum().

    Tokens whose target lies outside the vocabulary, or whose weight is 0, do not count: loss 0, no gradient.  dh or dw may be
    None.  workspace: ``head_workspace_bytes(h, w, piece=piece)`` bytes."""
    sizes, target_at, weight_at, out = _head(h, w, loss, dh, dw, weight, target)
    iwp._check(iwp._hot().iwp_head_cross_entropy(*sizes, target_at, weight_at, scale, piece, *out, workspace, iwp._bytes(workspace),
                                                 iwp._stream(stream)), "head_cross_entropy")


def head_distill(h, w, top_index, top_logit, loss, dh, dw, workspace, temperature: float = 1.0, soft: float = 1.0, target=None,
                 hard: float = 0.0, weight=None, scale: float = 1.0, piece: int = 0, stream=None):
    """loss[i] = weight[i] * (hard * CE_i + soft * temperature^2 * KL(q_i || softmax(h[i] w^T / temperature))), where q_i is the softmax
    of the teacher's top logits at that temperature; dh, dw = gradients of scale * loss.sum().

    top_index, top_logit: [tokens, top]; entries outside the vocabulary or with a logit of -inf are left out.  A token with neither a
    label nor an entry does not count.  workspace: ``head_workspace_bytes(h, w, top=top, piece=piece)`` bytes."""
    sizes, target_at, weight_at, out = _head(h, w, loss, dh, dw, weight, target)
    if top_index.dim() != 2:
        raise ValueError("top_index: a matrix is wanted")
    shape = (sizes[4], top_index.shape[1])
    iwp._check(iwp._hot().iwp_head_distill(*sizes, _packed(top_index, "top_index", shape, torch.int32),
                                           _packed(top_logit, "top_logit", shape, torch.float32), shape[1], temperature, soft, target_at,
                                           hard, weight_at, scale, piece, *out, workspace, iwp._bytes(workspace),
                                           iwp._stream(stream)), "head_distill")


def balance_workspace_bytes(tokens: int, experts: int) -> int:
    n = iwp.load().iwp_balance_workspace_bytes(tokens, experts)
    if n == 0:
        raise ValueError("sizes that the call refuses: %d tokens, %d experts" % (tokens, experts))
    return int(n)


def balance(x, chosen, loss, counts, dx, workspace, balance: float = 1.0, z: float = 0.0, keep=None, stream=None):
    """Balance of a router's choice.  x: [tokens, experts] logits, chosen: [tokens, slots] int32, keep: [tokens] uint8 or None.

    loss[0] = experts * sum_e share_e * mean(softmax(x)_e), loss[1] = mean(log sum exp(x)^2), over the tokens that count; counts[e]: slots
    given to expert e; dx = gradient of balance * loss[0] + z * loss[1].  A token does not count where keep is 0 or
    all its logits are -inf.  workspace: ``balance_workspace_bytes(tokens, experts)`` bytes."""
    if x.dim() != 2 or chosen.dim() != 2:
        raise ValueError("x and chosen: matrices are wanted")
    tokens, experts = x.shape
    code = _dtype(x, "x")
    x_at, ld_x = _matrix(x, "x", tokens, experts)
    dx_at, ld_dx = (None, 0) if dx is None else _matrix(dx, "dx", tokens, experts, x.dtype)
    slots = chosen.shape[1]
    iwp._check(iwp._hot().iwp_balance(x_at, ld_x, tokens, experts, code, _packed(chosen, "chosen", (tokens, slots), torch.int32), slots,
                                      _packed(keep, "keep", (tokens,), torch.uint8), balance, z, _packed(loss, "loss", (2,), torch.float32),
                                      _packed(counts, "counts", (experts,), torch.int32), dx_at, ld_dx, workspace,
                                      iwp._bytes(workspace), iwp._stream(stream)), "balance")
