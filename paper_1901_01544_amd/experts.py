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
    if x.dim() != 2 or chosen.dim() != 2:
        raise ValueError("x and chosen: matrices are wanted")
    tokens, experts = x.shape
    slots = chosen.shape[1]
    code = _dtype(x, "x")
    x_at, ld_x = _matrix(x, "x", tokens, experts)
    return (x_at, ld_x, tokens, experts, code), _packed(chosen, "chosen", (tokens, slots), torch.int32), slots


def route(x, chosen, weight, bias=None, scores: str = "softmax", groups: int = 1, top_groups: int = 0, group_top: int = 1,
          renormalise: bool = False, scale: float = 1.0, keep=None, stream=None):
    """chosen[i], weight[i]: the experts with the largest score + bias, the largest first, and scale * score of each (renormalise: over the sum of
    the token's chosen scores).

    x: [tokens, experts] logits; chosen: [tokens, slots] int32; weight: [tokens, slots] float32; scores: 'softmax' or 'sigmoid'; bias: [experts]
    float32, which weights have no part of.  groups: the experts in that many runs, of which a token may use the top_groups (0: all)
    with the largest sum of their group_top (1 or 2) best.  Slots without an expert, and those of tokens whose keep ([tokens] uint8) is 0,
    hold -1 and 0."""
    sizes, chosen_at, slots = _router(x, chosen)
    tokens, experts = sizes[2:4]
    iwp._check(iwp._hot().iwp_route(*sizes, _packed(bias, "bias", (experts,), torch.float32), _scores(scores), groups, top_groups or groups, group_top,
                                    int(bool(renormalise)), scale, _packed(keep, "keep", (tokens,), torch.uint8), chosen_at,
                                    _packed(weight, "weight", (tokens, slots), torch.float32), slots, iwp._stream(stream)), "route")


def route_gradient(x, chosen, dweight, dx, scores: str = "softmax", renormalise: bool = False, scale: float = 1.0, keep=None, plus=None,
                   stream=None):
    """dx = plus + the gradient of (weight * dweight).sum() with ``route``'s weights; chosen is a constant.

    dweight: [tokens, slots] float32; dx: of x's type and shape; plus: likewise, another gradient of x (``losses.balance``'s, say), which
    may be dx itself."""
    sizes, chosen_at, slots = _router(x, chosen)
    tokens, experts = sizes[2:4]
    plus_at, ld_plus = (None, 0) if plus is None else _matrix(plus, "plus", tokens, experts, x.dtype)
    dx_at, ld_dx = _matrix(dx, "dx", tokens, experts, x.dtype)
    iwp._check(iwp._hot().iwp_route_gradient(*sizes, chosen_at, _packed(dweight, "dweight", (tokens, slots), torch.float32), slots, _scores(scores),
                                             int(bool(renormalise)), scale, _packed(keep, "keep", (tokens,), torch.uint8), plus_at, ld_plus, dx_at,
                                             ld_dx, iwp._stream(stream)), "route_gradient")


def _sizes(x, w, chosen):
    """(tokens, slots, experts, in, out, type, whether x has a row for every slot)"""
    if chosen.dim() != 2 or w.dim() != 3 or x.dim() not in (2, 3):
        raise ValueError("x: [tokens, in] or [tokens, slots, in], w: [experts, out, in] and chosen: [tokens, slots] are wanted")
    tokens, slots = chosen.shape
    experts, out, width = w.shape
    if tuple(x.shape) != ((tokens, slots, width) if x.dim() == 3 else (tokens, width)):
        raise ValueError("x: %d tokens of %d slots, %d wide, are wanted, not %s" % (tokens, slots, width, tuple(x.shape)))
    return tokens, slots, experts, width, out, _dtype(x, "x"), int(x.dim() == 3)


def _rows(t, what: str, shape, dtype):
    """(address, elements from row to row) of a row for every token, or for every slot of it."""
    if tuple(t.shape) != shape or t.dtype != dtype:
        raise ValueError("%s: %s of shape %s is wanted, not %s of %s" % (what, dtype, shape, t.dtype, tuple(t.shape)))
    if t.dim() == 3:
        tokens, slots, width = shape
        # a slot's step is only there with two slots, a token's with two tokens
        if slots > 1 and tokens > 1 and t.stride(0) != slots * t.stride(1):
            raise ValueError("%s: rows of slots have to lie as far apart as rows of tokens' last and next first" % what)
        ld = t.stride(1) if slots > 1 else t.stride(0)
        if not t.is_cuda:
            raise ValueError("%s: a device tensor is wanted" % what)
        if t.stride(2) != 1 and width > 1:
            raise ValueError("%s: the elements of a row have to lie together" % what)
        return t.data_ptr(), max(ld, width) if tokens * slots <= 1 else ld
    return _matrix(t, what, *shape)


def _matrices(w, what: str, shape, dtype=None):
    """(address, elements from row to row, from matrix to matrix)."""
    if tuple(w.shape) != shape or (dtype is not None and w.dtype != dtype):
        raise ValueError("%s: %s of shape %s is wanted, not %s of %s" % (what, dtype or "a tensor", shape, w.dtype, tuple(w.shape)))
    if not w.is_cuda:
        raise ValueError("%s: a device tensor is wanted" % what)
    experts, rows, columns = shape
    if w.stride(2) != 1 and columns > 1:
        raise ValueError("%s: the elements of a row have to lie together" % what)
    ld = max(w.stride(1), columns) if rows <= 1 else w.stride(1)
    return w.data_ptr(), ld, w.stride(0) if experts > 1 else max(w.stride(0), rows * ld)


def product_workspace_bytes(x, w, chosen, gradient: bool = False) -> int:
    """Workspace of ``product``, or with gradient of ``product_gradient``, on these tensors."""
    tokens, slots, experts, width, out, code, by_slot = _sizes(x, w, chosen)
    at, ld, step = _matrices(w, "w", (experts, out, width), x.dtype)
    n = iwp.load().iwp_expert_product_workspace_bytes(tokens, slots, experts, width, out, code, at, ld, step, by_slot, int(bool(gradient)))
    if n == 0:
        raise ValueError("sizes that the products refuse: %d tokens of %d slots, %d experts of %d x %d" % (tokens, slots, experts, out, width))
    return int(n)


def product(x, w, chosen, y, workspace, stream=None):
    """y[i, k] = w[chosen[i, k]] @ x[i], or @ x[i, k]; zeros where chosen lies outside the experts.

    x: [tokens, in] or [tokens, slots, in]; w: [experts, out, in]; chosen: [tokens, slots] int32; y: [tokens, slots, out]; x, w and y of one type.
    workspace: ``product_workspace_bytes(x, w, chosen)`` bytes."""
    tokens, slots, experts, width, out, code, by_slot = _sizes(x, w, chosen)
    x_at, ld_x = _rows(x, "x", tuple(x.shape), x.dtype)
    y_at, ld_y = _rows(y, "y", (tokens, slots, out), x.dtype)
    iwp._check(iwp._hot().iwp_expert_product(x_at, ld_x, by_slot, *_matrices(w, "w", (experts, out, width), x.dtype), tokens, slots, experts, width, out,
                                             code, _packed(chosen, "chosen", (tokens, slots), torch.int32), y_at, ld_y, workspace, iwp._bytes(workspace),
                                             iwp._stream(stream)), "product")


def product_gradient(x, w, chosen, dy, dx, dw, workspace, stream=None):
    """dx, dw = gradients of (y * dy).sum() with ``product``'s y; either may be None.

    dy: [tokens, slots, out], of x's type; dx: of x's type and shape (a token's sum over its slots where x has one row a token); dw: [experts, out, in],
    of w's type or float32.  workspace: ``product_workspace_bytes(x, w, chosen, gradient=True)`` bytes."""
    tokens, slots, experts, width, out, code, by_slot = _sizes(x, w, chosen)
    x_at, ld_x = _rows(x, "x", tuple(x.shape), x.dtype)
    dy_at, ld_dy = _rows(dy, "dy", (tokens, slots, out), x.dtype)
    dx_at, ld_dx = (None, 0) if dx is None else _rows(dx, "dx", tuple(x.shape), x.dtype)
    dw_at, ld_dw, step_dw = (None, 0, 0) if dw is None else _matrices(dw, "dw", (experts, out, width))
    iwp._check(iwp._hot().iwp_expert_product_gradient(x_at, ld_x, by_slot, *_matrices(w, "w", (experts, out, width), x.dtype), tokens, slots, experts, width,
                                                      out, code, _packed(chosen, "chosen", (tokens, slots), torch.int32), dy_at, ld_dy, dx_at, ld_dx, dw_at,
                                                      ld_dw, step_dw, code if dw is None else _dtype(dw, "dw"), workspace, iwp._bytes(workspace),
                                                      iwp._stream(stream)), "product_gradient")
