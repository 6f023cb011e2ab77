"""The losses from their definitions in 64 bits, and how far binary32 sums and 16-bit roundings may take a result from them."""
import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}    # half a unit in the last place


def teacher(index, logit, t, vocab):
    """q over the vocabulary [tokens, vocab], sum q log q, and which tokens have an entry."""
    inside = (index >= 0) & (index < vocab) & (logit != float("-inf"))
    s = torch.where(inside, logit.double() / t, float("-inf"))
    any_ = inside.any(1)
    q = torch.where(any_[:, None], torch.softmax(torch.where(any_[:, None], s, 0.0), 1), 0.0)
    q = torch.where(inside, q, 0.0)
    dense = torch.zeros(index.shape[0], vocab, dtype=torch.float64, device=index.device)
    dense.scatter_add_(1, torch.where(inside, index, 0).long(), q)
    # an index that occurs twice counts entry by entry in the loss: sum q log q over entries
    entropy = torch.where(q > 0, q * torch.log(torch.where(q > 0, q, 1.0)), 0.0).sum(1)
    return dense, entropy, any_


class Head:
    """Results and error bounds of the head's losses; t: temperature, hard / soft: the parts' weights."""

    def __init__(self, h, w, target=None, index=None, logit=None, t=1.0, hard=1.0, soft=0.0, weight=None, scale=1.0):
        T, V = h.shape[0], w.shape[0]
        dev, kind = h.device, h.dtype
        a = torch.ones(T, dtype=torch.float64, device=dev) if weight is None else weight.double()
        label = torch.full((T,), -1, device=dev) if target is None else target.long()
        has_label = (label >= 0) & (label < V)
        q = torch.zeros(T, V, dtype=torch.float64, device=dev)
        entropy = torch.zeros(T, dtype=torch.float64, device=dev)
        has_entry = torch.zeros(T, dtype=torch.bool, device=dev)
        if index is not None:
            q, entropy, has_entry = teacher(index, logit, t, V)
        counts = (a != 0) & ((has_label & (hard != 0)) | (has_entry & (soft != 0)))
        self.counts = counts
        rows = counts.nonzero().squeeze(1)
        H, W = h.double()[rows], w.double()
        z = H @ W.t()
        lse, lse_t = torch.logsumexp(z, 1), torch.logsumexp(z / t, 1)
        p, p_t = (z - lse[:, None]).exp(), (z / t - lse_t[:, None]).exp()
        y = torch.where(has_label, label, 0)[rows]
        one = torch.zeros_like(z).scatter_(1, y[:, None], 1.0)
        ch = torch.where(has_label, a, 0.0)[rows] * hard
        cs = torch.where(has_entry, a, 0.0)[rows] * soft
        ce = lse - (z * one).sum(1)
        kl = entropy[rows] - (q[rows] * z).sum(1) / t + lse_t
        self.loss = torch.zeros(T, dtype=torch.float64, device=dev)
        self.loss[rows] = ch * ce + cs * t * t * kl
        # |z| is off by binary32 sums over the width (and by 2^-21 of the operands where they are split)
        reach = H.norm(dim=1, keepdim=True) * W.norm(dim=1)
        off_z = 2.0 ** -20 * reach.amax(1)
        self.loss_off = torch.zeros_like(self.loss)
        self.loss_off[rows] = (ch.abs() * (2 * off_z + 2.0 ** -20 * (1 + lse.abs() + z.abs().amax(1)))
                               + cs.abs() * t * t * (2 * off_z / t + 2.0 ** -20 * (1 + entropy[rows].abs() + lse_t.abs() + z.abs().amax(1) / t)))
        label_part, soft_part = ch[:, None] * (p - one), cs[:, None] * t * (p_t - q[rows])
        dz = scale * (label_part + soft_part)
        # each term of dz: exponentials of logits that are off, then one rounding to the operands' type
        grown = abs(scale) * (ch.abs()[:, None] * (p + one) + cs.abs()[:, None] * t * (p_t + q[rows]))
        off = grown * (2 * off_z[:, None] + 2.0 ** -19 * (1 + z.abs()))
        if kind != torch.float32:
            off = off + UNIT[kind] * dz.abs()
        if kind == torch.bfloat16:                          # kept as differences to a largest logit in fp16
            off = off + 2.0 ** -11 * grown * (z.amax(1, keepdim=True) - z)
        most = abs(scale) * (ch.abs() + cs.abs() * t).max() if rows.numel() else 0.0
        off = off + 2.0 ** -38 * most                       # where fp16 ends
        self.dh = torch.zeros(h.shape, dtype=torch.float64, device=dev)
        self.dh_off = torch.zeros_like(self.dh)
        self.dh[rows] = dz @ W
        self.dh_off[rows] = off @ W.abs() + 2.0 ** -20 * (dz.abs() @ W.abs())
        self.dw = dz.t() @ H
        self.dw_off = off.t() @ H.abs() + 2.0 ** -20 * (dz.abs().t() @ H.abs())

    def check(self, loss, dh, dw):
        near("loss", loss, self.loss, self.loss_off)
        if dh is not None:
            near("dh", dh, self.dh, self.dh_off)
            assert (dh[~self.counts] == 0).all()
        if dw is not None:
            near("dw", dw, self.dw, self.dw_off)


def near(what, got, want, off):
    tiny = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}[got.dtype]
    allowed = off + UNIT[got.dtype] * want.abs() + tiny
    d = (got.double() - want).abs()
    bad = ~(d <= allowed)
    assert not bad.any(), "%s: %d of %d values off, worst %.3g where %.3g is allowed (value %.6g)" % (
        what, int(bad.sum()), bad.numel(), d[bad].max().item(), allowed[bad][d[bad].argmax()].item(),
        want[bad][d[bad].argmax()].item())


class Balance:
    def __init__(self, x, chosen, balance, z, keep=None):
        T, E = x.shape
        K = chosen.shape[1]
        dev = x.device
        counts = torch.ones(T, dtype=torch.bool, device=dev) if keep is None else keep != 0
        counts = counts & ~(x == float("-inf")).all(1)
        rows = counts.nonzero().squeeze(1)
        X = x.double()[rows]
        n = rows.numel()
        self.counts = torch.zeros(E, dtype=torch.int32, device=dev)
        self.loss = torch.zeros(2, dtype=torch.float64, device=dev)
        self.dx = torch.zeros(x.shape, dtype=torch.float64, device=dev)
        self.loss_off, self.dx_off = torch.zeros_like(self.loss), torch.zeros_like(self.dx)
        if n == 0:
            return
        c = chosen.long()[rows].reshape(-1)
        c = c[(c >= 0) & (c < E)]
        self.counts = torch.bincount(c, minlength=E).to(torch.int32)
        share = self.counts.double() / (n * K)
        L = torch.logsumexp(X, 1)
        p = (X - L[:, None]).exp()
        self.loss = torch.stack([E * (share * p.mean(0)).sum(), (L * L).mean()])
        size = X.masked_fill(X == float("-inf"), 0.0).abs().amax(1, keepdim=True)
        rel = 2.0 ** -20 * (1 + size)                       # exponentials of binary32 differences, sums in binary32
        self.loss_off = torch.stack([E * (share * (p * rel).mean(0)).sum() * 2, (2.0 ** -19 * (1 + L * L)).mean()])
        inner = p @ share
        cb, cz = balance * E / n, 2.0 * z / n
        self.dx[rows] = p * (cb * (share - inner[:, None]) + cz * L[:, None])
        self.dx_off[rows] = p * (rel * (abs(cb) * (share + 2 * inner[:, None]) + abs(cz) * (1 + L.abs())[:, None]))

    def check(self, loss, counts, dx):
        assert torch.equal(counts, self.counts)
        near("loss", loss, self.loss, self.loss_off)
        if dx is not None:
            near("dx", dx, self.dx, self.dx_off)
