"""The routed layer's operators from their definitions in 64 bits, and how far binary32 sums and roundings of the result may take a value."""
import torch

from loss_reference import near


def scores_of(x, scores):
    """Scores in 64 bits of logits in 64 bits; -inf has none."""
    dead = x == float("-inf")
    if scores == "softmax":
        s = torch.softmax(torch.where(dead.all(1, keepdim=True), 0.0, x), 1)
    else:
        s = torch.sigmoid(x)
    return torch.where(dead, 0.0, s)


class Route:
    """chosen, weight and its bound."""

    def __init__(self, x, slots, bias=None, scores="softmax", groups=1, top_groups=0, group_top=1, renormalise=False, scale=1.0, keep=None):
        X = x.double()
        T, E = X.shape
        top_groups = top_groups or groups
        by_score = bias is not None or (top_groups < groups and group_top == 2)
        c = X.clone()
        if by_score:
            c = scores_of(X, scores) + (0.0 if bias is None else bias.double())
        c = torch.where((X == float("-inf")) | torch.isnan(X) | torch.isnan(c), float("-inf"), c)
        if keep is not None:
            c[keep == 0] = float("-inf")
        if top_groups < groups:
            size = E // groups
            best = c.view(T, groups, size).sort(dim=2, descending=True).values[:, :, :group_top]
            none = best[:, :, 0] == float("-inf")
            total = torch.where(none, float("-inf"), torch.where(best == float("-inf"), 0.0, best).sum(2))
            order = total.sort(dim=1, descending=True, stable=True).indices[:, :top_groups]
            inside = torch.zeros(T, groups, dtype=torch.bool, device=x.device).scatter_(1, order, True)
            c = torch.where(inside.repeat_interleave(size, 1), c, float("-inf"))
        value, at = c.sort(dim=1, descending=True, stable=True)
        there = value[:, :slots] > float("-inf")
        at = at[:, :slots]
        self.chosen = torch.where(there, at, -1).to(torch.int32)
        s = scores_of(X, scores)
        picked = torch.where(there, s.gather(1, at), 0.0)
        if renormalise:
            total = picked.sum(1, keepdim=True)
            picked = picked / torch.where(total == 0, 1.0, total)
        self.weight = scale * picked
        # exponentials of binary32 differences (off by 2^-24 of the difference, then 2^-22), a sum of at most 16 + 6 steps, a quotient
        size = torch.where(torch.isfinite(X), X.abs(), 0.0).amax(1, keepdim=True)
        self.off = 2.0 ** -19 * (1 + size) * self.weight.abs()

    def check(self, chosen, weight):
        assert torch.equal(chosen, self.chosen)
        near("weight", weight, self.weight, self.off)


class RouteGradient:
    def __init__(self, x, chosen, dweight, scores="softmax", renormalise=False, scale=1.0, keep=None, plus=None):
        X = x.double()
        T, E = X.shape
        there = (chosen >= 0) & (chosen < E)
        if keep is not None:
            there = there & (keep != 0)[:, None]
        at = torch.where(there, chosen, 0).long()
        dw = torch.where(there, dweight.double(), 0.0) * scale
        s = scores_of(X, scores)
        picked = torch.where(there, s.gather(1, at), 0.0)
        total = picked.sum(1, keepdim=True) if renormalise else torch.ones(T, 1, dtype=torch.float64, device=x.device)
        v = picked / torch.where(total == 0, 1.0, total)
        # of slot k: d weight_l / d log s_k = v_k [k = l] - v_k v_l with the renormalisation, v_k [k = l] without
        by_log = v * dw - (v * (v * dw).sum(1, keepdim=True) if renormalise else 0.0)
        grown = v * dw.abs() + (v * (v * dw).abs().sum(1, keepdim=True) if renormalise else 0.0)
        zero = torch.zeros(T, E, dtype=torch.float64, device=x.device)
        of, of_grown = zero.scatter_add(1, at, by_log), zero.scatter_add(1, at, grown)
        if scores == "sigmoid":                             # d log s_j / d x_j = 1 - s_j
            self.dx, grown = of * torch.sigmoid(-X), of_grown * torch.sigmoid(-X)
        elif renormalise:                                   # d log s_k / d x_j = [k = j] - s_j, and the by_log sum to nothing
            self.dx, grown = of, of_grown
        else:
            self.dx, grown = of - s * by_log.sum(1, keepdim=True), of_grown + s * grown.sum(1, keepdim=True)
        size = torch.where(torch.isfinite(X), X.abs(), 0.0).amax(1, keepdim=True)
        self.off = 2.0 ** -18 * (1 + size) * grown          # as the weights, twice: q / sum times a difference of dweight and a sum over q
        if plus is not None:
            self.off = self.off + 2.0 ** -24 * (plus.double().abs() + self.dx.abs())
            self.dx = self.dx + plus.double()

    def check(self, dx):
        near("dx", dx, self.dx, self.off)


class Experts:
    """y and the gradients of products with every expert's matrix, row by row of the slots."""

    def __init__(self, x, w, chosen, dy=None):
        T, K = chosen.shape
        E, F, D = w.shape
        by_slot = x.dim() == 3
        X = (x if by_slot else x[:, None].expand(T, K, D)).reshape(T * K, D).double()
        c = chosen.reshape(-1).long()
        self.nobody = ((c < 0) | (c >= E)).view(T, K)
        zeros = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device=x.device)  # noqa: E731
        y, y_off = zeros(T * K, F), zeros(T * K, F)
        dx, dx_off, self.dw, self.dw_off = zeros(T * K, D), zeros(T * K, D), zeros(E, F, D), zeros(E, F, D)
        d = None if dy is None else dy.reshape(T * K, F).double()
        for e in range(E):
            rows = (c == e).nonzero().squeeze(1)
            if not rows.numel():
                continue
            W = w[e].double()
            y[rows] = X[rows] @ W.t()
            y_off[rows] = 2.0 ** -20 * (X[rows].abs() @ W.abs().t())           # sums in binary32
            if d is not None:
                dx[rows] = d[rows] @ W
                dx_off[rows] = 2.0 ** -20 * (d[rows].abs() @ W.abs())
                self.dw[e] = d[rows].t() @ X[rows]
                self.dw_off[e] = 2.0 ** -20 * (d[rows].abs().t() @ X[rows].abs())
        self.y, self.y_off = y.view(T, K, F), y_off.view(T, K, F)
        dx, dx_off = dx.view(T, K, D), dx_off.view(T, K, D)
        if not by_slot:
            dx_off = dx_off.sum(1) + 2.0 ** -23 * K * dx.abs().sum(1)
            dx = dx.sum(1)
        self.dx, self.dx_off = dx, dx_off

    def check(self, y):
        near("y", y, self.y, self.y_off)
        assert (y[self.nobody] == 0).all()

    def check_gradient(self, dx, dw):
        if dx is not None:
            near("dx", dx, self.dx, self.dx_off)
        if dw is not None:
            near("dw", dw, self.dw, self.dw_off)
