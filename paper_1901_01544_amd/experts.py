"""Operators of a layer with routed experts: binding of ``include/iwp_experts.h``.

    experts.route               experts for every token from a router's logits, with their weights
    experts.route_gradient      the logits' gradient from the weights'
    experts.product             every slot's row through the matrix of the expert chosen for it
    experts.product_gradient    the rows' and the matrices' gradients

Conventions are those of ``losses``: outputs and workspaces are the caller's, rows of matrices may be strided, the calls only enqueue kernels
on ``stream``, and a matrix's gradient may be a view into the flat binary32 gradients of ``iwp.step_segmented`` whatever the operands' type is.
``chosen`` is what ``losses.balance`` takes, and its gradient of the logits can be handed to ``route_gradient`` as ``plus``.
"""
from __future__ import annotations

import torch

from . import iwp
from .losses import _dtype, _matrix, _packed

SOFTMAX, SIGMOID = 0, 1
_SCORES = {"softmax": SOFTMAX, "sigmoid": SIGMOID}


def _scores(scores: str) -> int:
    code = _SCORES.get(scores)
    if code is None:
        raise ValueError("scores: 'softmax' or 'sigmoid' is wanted, not %r" % (scores,))
    return code


def _router(x, chosen):
    """Sizes of the logits, of the slots; where chosen is."""
    size, slots = x.shape, chosen.shape
    if len(size) != 2 or len(slots) != 2:
        raise ValueError("x and chosen: matrices are wanted")
    tokens, experts = size
    if slots[0] != tokens:
        raise ValueError("chosen: a row for each of %d tokens is wanted, not %s" % (tokens, tuple(slots)))
    code = _dtype(x, "x")
    return (*_matrix(x, "x", tokens, experts), tokens, experts, code), slots, _packed(chosen, "chosen", slots, torch.int32)


def route(x, chosen, weight, bias=None, scores: str = "softmax", groups: int = 1, top_groups: int = 0, group_top: int = 1,
          renormalise: bool = False, scale: float = 1.0, keep=None, stream=None):
    """chosen[i], weight[i]: the experts with the largest score + bias (without a bias: the largest logits), the largest first, and scale * score of each (renormalise: over the sum of
    the token's chosen scores).

    x: [tokens, experts] logits; chosen: [tokens, slots] int32; weight: [tokens, slots] float32; scores: 'softmax' or 'sigmoid'; bias: [experts]
    float32, which weights have no part of.  groups: the experts in that many runs, of which a token may use the top_groups (0: all)
    with the largest sum of their group_top (1 or 2) best.  Slots without an expert, and those of tokens whose keep ([tokens] uint8) is 0,
    hold -1 and 0."""
    sizes, slots, chosen_at = _router(x, chosen)
    iwp._check(iwp._hot().iwp_route(*sizes, bias if bias is None else _packed(bias, "bias", (sizes[3],), torch.float32), _scores(scores), groups,
                                    top_groups or groups, group_top, 1 if renormalise else 0, scale,
                                    keep if keep is None else _packed(keep, "keep", (sizes[2],), torch.uint8), chosen_at,
                                    _packed(weight, "weight", slots, torch.float32), slots[1], iwp._stream(stream)), "route")


def route_gradient(x, chosen, dweight, dx, scores: str = "softmax", renormalise: bool = False, scale: float = 1.0, keep=None, plus=None,
                   stream=None):
    """dx = plus + the gradient of (weight * dweight).sum() with ``route``'s weights; chosen is a constant.

    dweight: [tokens, slots] float32; dx: of x's type and shape; plus: likewise, another gradient of x (``losses.balance``'s, say), which
    may be dx itself."""
    sizes, slots, chosen_at = _router(x, chosen)
    tokens, experts = sizes[2:4]
    plus_at, ld_plus = (None, 0) if plus is None else _matrix(plus, "plus", tokens, experts, x.dtype)
    iwp._check(iwp._hot().iwp_route_gradient(*sizes, chosen_at, _packed(dweight, "dweight", slots, torch.float32), slots[1], _scores(scores),
                                             1 if renormalise else 0, scale, keep if keep is None else _packed(keep, "keep", (tokens,), torch.uint8),
                                             plus_at, ld_plus, *_matrix(dx, "dx", tokens, experts, x.dtype), iwp._stream(stream)), "route_gradient")


def _sizes(x, w, chosen):
    """(tokens, slots, experts, in, out, type), whether x has a row for every slot."""
    size, matrices, slots = x.shape, w.shape, chosen.shape
    if len(slots) != 2 or len(matrices) != 3 or len(size) not in (2, 3):
        raise ValueError("x: [tokens, in] or [tokens, slots, in], w: [experts, out, in] and chosen: [tokens, slots] are wanted")
    by_slot = len(size) == 3
    if size[:-1] != slots[:2 if by_slot else 1] or size[-1] != matrices[2]:
        raise ValueError("x: %d tokens of %d slots, %d wide, are wanted, not %s" % (*slots, matrices[2], tuple(size)))
    return (slots[0], slots[1], matrices[0], matrices[2], matrices[1], _dtype(x, "x")), 1 if by_slot else 0


def _rows(t, what: str, shape, dtype):
    """(address, elements from row to row) of a row for every token, or for every slot of it."""
    if t.shape != shape or t.dtype != dtype:
        raise ValueError("%s: %s of shape %s is wanted, not %s of %s" % (what, dtype, tuple(shape), t.dtype, tuple(t.shape)))
    if len(shape) == 2:
        return _matrix(t, what, *shape)
    tokens, slots, width = shape
    of_token, ld, step = t.stride()
    if slots == 1:
        ld = of_token
    elif tokens > 1 and of_token != slots * ld:                      # a token's step is only there with two tokens
        raise ValueError("%s: a token's last row and the next one's first have to lie as far apart as rows of a token" % what)
    if not t.is_cuda:
        raise ValueError("%s: a device tensor is wanted" % what)
    if step != 1 and width > 1:
        raise ValueError("%s: the elements of a row have to lie together" % what)
    return t.data_ptr(), max(ld, width) if tokens * slots <= 1 else ld


def _matrices(w, what: str, shape, dtype=None):
    """(address, elements from row to row, from matrix to matrix)."""
    if w.shape != shape or (dtype is not None and w.dtype != dtype):
        raise ValueError("%s: %s of shape %s is wanted, not %s of %s" % (what, dtype or "a tensor", tuple(shape), w.dtype, tuple(w.shape)))
    if not w.is_cuda:
        raise ValueError("%s: a device tensor is wanted" % what)
    experts, rows, columns = shape
    step, ld, one = w.stride()
    if one != 1 and columns > 1:
        raise ValueError("%s: the elements of a row have to lie together" % what)
    if rows <= 1:
        ld = max(ld, columns)
    return w.data_ptr(), ld, step if experts > 1 else max(step, rows * ld)


def product_workspace_bytes(x, w, chosen, gradient: bool = False) -> int:
    """Workspace of ``product``, or with gradient of ``product_gradient``, on these tensors."""
    sizes, by_slot = _sizes(x, w, chosen)
    n = iwp.load().iwp_expert_product_workspace_bytes(*sizes, *_matrices(w, "w", w.shape, x.dtype), by_slot, int(bool(gradient)))
    if n == 0:
        raise ValueError("sizes that the products refuse: %d tokens of %d slots, %d experts of %d x %d" % (*sizes[:3], sizes[4], sizes[3]))
    return int(n)


def product(x, w, chosen, y, workspace, stream=None):
    """y[i, k] = w[chosen[i, k]] @ x[i], or @ x[i, k]; zeros where chosen lies outside the experts.

    x: [tokens, in] or [tokens, slots, in]; w: [experts, out, in]; chosen: [tokens, slots] int32; y: [tokens, slots, out]; x, w and y of one type.
    workspace: ``product_workspace_bytes(x, w, chosen)`` bytes."""
    sizes, by_slot = _sizes(x, w, chosen)
    kind = x.dtype
    iwp._check(iwp._hot().iwp_expert_product(*_rows(x, "x", x.shape, kind), by_slot, *_matrices(w, "w", w.shape, kind), *sizes,
                                             _packed(chosen, "chosen", chosen.shape, torch.int32), *_rows(y, "y", (sizes[0], sizes[1], sizes[4]), kind),
                                             workspace, iwp._bytes(workspace), iwp._stream(stream)), "product")


def product_gradient(x, w, chosen, dy, dx, dw, workspace, stream=None):
    """dx, dw = gradients of (y * dy).sum() with ``product``'s y; either may be None.

    dy: [tokens, slots, out], of x's type; dx: of x's type and shape (a token's sum over its slots where x has one row a token); dw: [experts, out, in],
    of w's type or float32.  workspace: ``product_workspace_bytes(x, w, chosen, gradient=True)`` bytes."""
    sizes, by_slot = _sizes(x, w, chosen)
    kind = x.dtype
    dx_at = (None, 0) if dx is None else _rows(dx, "dx", x.shape, kind)
    dw_at = (None, 0, 0, sizes[5]) if dw is None else (*_matrices(dw, "dw", w.shape), _dtype(dw, "dw"))
    iwp._check(iwp._hot().iwp_expert_product_gradient(*_rows(x, "x", x.shape, kind), by_slot, *_matrices(w, "w", w.shape, kind), *sizes,
                                                      _packed(chosen, "chosen", chosen.shape, torch.int32),
                                                      *_rows(dy, "dy", (sizes[0], sizes[1], sizes[4]), kind), *dx_at, *dw_at, workspace,
                                                      iwp._bytes(workspace), iwp._stream(stream)), "product_gradient")
