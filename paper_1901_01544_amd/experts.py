"""Operators of a layer with routed experts: binding of ``include/iwp_experts.h``.

    experts.route               experts for every token from a router's logits, with their weights
    experts.route_gradient      the logits' gradient from the weights'

Conventions are those of ``losses``: outputs are the caller's, rows of matrices may be strided, the calls only enqueue kernels on ``stream``.
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
