"""A training step with routed experts, from the router's logits to the gradients that are compressed.

``route`` / ``route_gradient`` cases: logits [T, E] of a router; what comes back is the experts chosen for every token with their
weights, or the gradient of the logits.  ``product`` / ``product_gradient`` cases: every token's rows through the matrices of the
experts chosen for it; what comes back is the rows' products, or the gradients of the tokens and of all experts' matrices.  ``clip``
cases: the flat gradients of W workers; what comes back is their norms and the gradients scaled to a largest norm.
"""
from __future__ import annotations

import math

import torch

own = False             # True: the framework's kernels; False: the plain forms

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # the batch of the example's language model: launches are all there is
        {"name": "route_few", "op": "route", "T": 200, "E": 8, "K": 2, "type": "f32", "scores": "softmax", "bias": False,
         "groups": 1, "top_groups": 1, "group_top": 1, "renormalise": True, "scale": 1.0, "masked": 0.0, "ignored": 0.125},
        # an ordinary router in a padded batch
        {"name": "route_step", "op": "route", "T": 16384, "E": 64, "K": 4, "type": "bf16", "scores": "softmax", "bias": False,
         "groups": 1, "top_groups": 1, "group_top": 1, "renormalise": False, "scale": 1.0, "masked": 0.1, "ignored": 0.2},
        # many experts over eight groups of machines, balanced by a bias, a long batch
        {"name": "route_large", "op": "route", "T": 131072, "E": 256, "K": 8, "type": "f32", "scores": "sigmoid", "bias": True,
         "groups": 8, "top_groups": 4, "group_top": 2, "renormalise": True, "scale": 2.5, "masked": 0.0, "ignored": 0.0},
        # the ordinary router's way back, on top of the balance loss's gradient
        {"name": "route_gradient_step", "op": "route_gradient", "T": 16384, "E": 64, "K": 4, "type": "bf16", "scores": "softmax",
         "renormalise": False, "scale": 1.0, "plus": True, "nobody": 0.05, "ignored": 0.2},
        # the large router's way back
        {"name": "route_gradient_large", "op": "route_gradient", "T": 131072, "E": 256, "K": 8, "type": "f32",
         "scores": "sigmoid", "renormalise": True, "scale": 2.5, "plus": False, "nobody": 0.0, "ignored": 0.0},
        # one token, eight of its experts: the matrices' bytes
        {"name": "product_single", "op": "product", "T": 1, "K": 8, "E": 64, "in": 2048, "out": 1024, "type": "bf16",
         "per_slot": False, "nobody": 0.0},
        # binary32, as the flat buffers hold weights; odd sizes, a third of the slots empty (experts that were full)
        {"name": "product_odd", "op": "product", "T": 1021, "K": 3, "E": 17, "in": 1001, "out": 777, "type": "f32",
         "per_slot": True, "nobody": 0.33},
        # an ordinary step's first product of eight wide experts
        {"name": "product_step", "op": "product", "T": 8192, "K": 2, "E": 8, "in": 2048, "out": 4096, "type": "bf16",
         "per_slot": False, "nobody": 0.0},
        # a small model's, half precision, a matrix per slot's own row
        {"name": "product_gradient_odd", "op": "product_gradient", "T": 333, "K": 2, "E": 8, "in": 513, "out": 640, "type": "f16",
         "per_slot": True, "nobody": 0.05},
        # an ordinary step of many narrow experts
        {"name": "product_gradient_step", "op": "product_gradient", "T": 8192, "K": 4, "E": 64, "in": 2048, "out": 1024,
         "type": "bf16", "per_slot": False, "nobody": 0.0},
        # a small perceptron's four workers
        {"name": "clip_small", "op": "clip", "W": 4, "sizes": "200704 256 32768 128 1280 10", "align": 64, "scale": 1.0},
        # the layer table of a large convolutional classifier, eight workers; the losses were scaled for half precision
        {"name": "clip_large", "op": "clip", "W": 8, "align": 64, "scale": 1.0 / 65536,
         "sizes": "34848 96 614400 256 884736 384 1327104 384 884736 256 37748736 4096 16777216 4096 4096000 1000"},
    ]


def _spread(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    op = rng.choice(["route", "route", "route_gradient", "product", "product", "product_gradient", "clip"])
    if op == "clip":
        most = 61_000_000
        sizes = []
        for _ in range(_spread(rng, 1, 200)):
            n = _spread(rng, 1, 20_000_000)
            if sum(sizes) + n <= most:
                sizes.append(n)
        sizes = sizes or [_spread(rng, 1, 1_000_000)]
        return {"op": op, "W": rng.randint(1, 8), "sizes": " ".join(map(str, sizes)), "align": rng.choice([1, 4, 64]),
                "scale": rng.choice([1.0, 1.0, 1.0 / 65536, 0.125])}
    kind = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op in ("route", "route_gradient"):
        T, E = _spread(rng, 1, 131072), _spread(rng, 4, 256)
        case = {"op": op, "T": T, "E": E, "type": kind, "scores": rng.choice(["softmax", "sigmoid"]),
                "renormalise": rng.random() < 0.5, "scale": rng.choice([1.0, 1.0, 2.5]), "ignored": rng.choice([0.0, 0.05, 0.2, 0.5])}
        if op == "route":
            groups = rng.choice([1, 1, 2, 4, 8])
            E = max(groups * 2, E // groups * groups)
            top_groups = rng.randint(1, groups)
            case.update(E=E, bias=rng.random() < 0.5, groups=groups, top_groups=top_groups, group_top=rng.choice([1, 2]),
                        masked=rng.choice([0.0, 0.0, 0.1, 0.6]), K=rng.randint(1, min(8, E // groups * top_groups)))
        else:
            case.update(K=rng.randint(1, min(8, E)), plus=rng.random() < 0.5, nobody=rng.choice([0.0, 0.05, 0.5]))
        return case
    T, K, E = _spread(rng, 1, 8192), rng.randint(1, 8), _spread(rng, 4, 64)
    D, F = _spread(rng, 256, 4096), _spread(rng, 256, 4096)
    if rng.random() < 0.6:                      # widths are round more often than not
        D, F = max(256, D // 128 * 128), max(256, F // 128 * 128)
    # operations and matrices of the largest listed case at most; binary32 costs eight times as much
    most = 8192 * 2 * 2048 * 4096 // (8 if kind == "f32" else 1) // (2 if op == "product_gradient" else 1)
    while T * K * D * F > most:
        T, K = max(1, T // 2), max(1, K - 1)
    E = max(2, min(E, 64 * 2048 * 1024 // (D * F)))
    return {"op": op, "T": T, "K": min(K, E), "E": E, "in": D, "out": F, "type": kind, "per_slot": rng.random() < 0.4,
            "nobody": rng.choice([0.0, 0.05, 0.33])}


# ------------------------------------------------------------------ inputs

def _kept(case, gen):
    """Which tokens count: a run at the start of every stretch of some hundred tokens does not (a prompt, or padding)."""
    T = case["T"]
    length = max(1, min(T, 257))
    phase = torch.rand((), generator=gen, device=DEVICE) * length
    return ((torch.arange(T, device=DEVICE) + phase) % length) >= case["ignored"] * length


def _logits(case, gen):
    """Logits of a router that likes some experts more than others."""
    T, E = case["T"], case["E"]
    return (torch.randn(T, E, generator=gen, device=DEVICE) + 0.7 * torch.randn(E, generator=gen, device=DEVICE)).to(TYPES[case["type"]])


def _choice(case, gen):
    """Distinct experts for every token, some liked more than others, and slots that nobody got."""
    T, E, K = case["T"], case["E"], case["K"]
    liked = torch.randn(T, E, generator=gen, device=DEVICE) + 0.5 * torch.randn(E, generator=gen, device=DEVICE)
    chosen = liked.topk(K, dim=1).indices.to(torch.int32)
    nobody = torch.rand(T, K, generator=gen, device=DEVICE) < case["nobody"]
    return torch.where(nobody, -1, chosen)


def _rows(case):
    """(offset, elements) of the tensors in a flat buffer, and its length."""
    rows, at = [], 0
    for n in map(int, case["sizes"].split()):
        rows.append((at, n))
        at = (at + n + case["align"] - 1) // case["align"] * case["align"]
    return rows, at


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(6271 * int(seed) + 29)
    s = {"case": case}
    if case["op"] == "clip":
        rows, flat = _rows(case)
        # tensors' gradients of different size (fan-in), workers louder and quieter than the largest norm
        g = [torch.zeros(flat, device=DEVICE) for _ in range(case["W"])]
        loud = (2.0 * torch.rand(case["W"], generator=gen, device=DEVICE) - 1.0).exp2()
        expected = 0.0
        for j, (at, n) in enumerate(rows):
            size = 1e-3 * 2.0 ** -(j % 5)
            expected += n * size * size
            for p, flat_p in enumerate(g):
                flat_p[at:at + n].normal_(0.0, size / case["scale"], generator=gen).mul_(loud[p])
        s.update(g=g, out=[torch.zeros_like(x) for x in g], norm=torch.empty(case["W"], device=DEVICE), rows=rows,
                 max_norm=math.sqrt(expected))
        if own:
            from paper_1901_01544_amd import clipping
            s["tensors"] = clipping.Tensors(rows)
            s["workspace"] = torch.empty(s["tensors"].workspace_bytes(case["W"]), dtype=torch.uint8, device=DEVICE)
        return s
    T, E, K, kind = case["T"], case["E"], case["K"], TYPES[case["type"]]
    if case["op"] == "route":
        x = _logits(case, gen)
        if case["masked"]:                      # experts that are out of reach for a token
            x = torch.where(torch.rand(T, E, generator=gen, device=DEVICE) < case["masked"], float("-inf"), x)
        s.update(x=x, keep=_kept(case, gen).to(torch.uint8), chosen=torch.empty(T, K, dtype=torch.int32, device=DEVICE),
                 weight=torch.empty(T, K, device=DEVICE), bias=None)
        if case["bias"]:                        # as the rule that moves it by small steps leaves it
            s["bias"] = 0.001 * torch.randint(-40, 41, (E,), generator=gen, device=DEVICE).float()
        return s
    if case["op"] == "route_gradient":
        s.update(x=_logits(case, gen), chosen=_choice(case, gen), keep=_kept(case, gen).to(torch.uint8), plus=None,
                 dweight=0.01 * torch.randn(T, K, generator=gen, device=DEVICE))
        if case["plus"]:
            s["plus"] = (0.001 * torch.randn(T, E, generator=gen, device=DEVICE)).to(kind)
        s["dx"] = torch.empty_like(s["x"])
        return s
    D, F = case["in"], case["out"]
    shape = (T, K, D) if case["per_slot"] else (T, D)
    s["x"] = torch.randn(shape, generator=gen, device=DEVICE).to(kind)
    s["w"] = torch.empty(E, F, D, device=DEVICE).normal_(0.0, D ** -0.5, generator=gen).to(kind)
    s["chosen"] = _choice(case, gen)
    if case["op"] == "product":
        s["y"] = torch.empty(T, K, F, dtype=kind, device=DEVICE)
    else:
        s["dy"] = (0.02 * torch.randn(T, K, F, generator=gen, device=DEVICE)).to(kind)
        s["dx"] = torch.empty_like(s["x"])
        s["dw"] = torch.empty(E, F, D, device=DEVICE)          # binary32: a view of the flat gradients
    if own:
        from paper_1901_01544_amd import experts
        s["workspace"] = torch.empty(experts.product_workspace_bytes(s["x"], s["w"], s["chosen"], gradient=case["op"] != "product"),
                                     dtype=torch.uint8, device=DEVICE)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    case = s["case"]
    return (_run_own if own else _run_plain)(case["op"], case, s)


def _run_own(op, case, s):
    from paper_1901_01544_amd import clipping, experts
    if op == "route":
        experts.route(s["x"], s["chosen"], s["weight"], bias=s["bias"], scores=case["scores"], groups=case["groups"],
                      top_groups=case["top_groups"], group_top=case["group_top"], renormalise=case["renormalise"],
                      scale=case["scale"], keep=s["keep"])
        return {"chosen": s["chosen"], "weight": s["weight"]}
    if op == "route_gradient":
        experts.route_gradient(s["x"], s["chosen"], s["dweight"], s["dx"], scores=case["scores"], renormalise=case["renormalise"],
                               scale=case["scale"], keep=s["keep"], plus=s["plus"])
        return {"dx": s["dx"]}
    if op == "product":
        experts.product(s["x"], s["w"], s["chosen"], s["y"], s["workspace"])
        return {"y": s["y"]}
    if op == "product_gradient":
        experts.product_gradient(s["x"], s["w"], s["chosen"], s["dy"], s["dx"], s["dw"], s["workspace"])
        return {"dx": s["dx"], "dw": s["dw"]}
    clipping.clip(s["tensors"], s["g"], s["out"], s["norm"], s["workspace"], max_norm=s["max_norm"], scale=case["scale"])
    return {"norm": s["norm"], "out": s["out"]}


def _run_plain(op, case, s):
    if op == "route":
        return _plain_route(case, s)
    if op == "route_gradient":
        return _plain_route_gradient(case, s)
    if op == "product":
        return _plain_product(s)
    if op == "product_gradient":
        return _plain_product_gradient(s)
    return _plain_clip(case, s)


def _softmax(x):
    top = x.max(-1, keepdim=True).values
    e = (x - torch.where(top == float("-inf"), 0.0, top)).exp()
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total == 0, 1.0, total)


def _scores(x, scores):
    return _softmax(x) if scores == "softmax" else 1.0 / (1.0 + (-x).exp())


def _descending(values):
    """Positions by value, the largest first, the lowest position first where values are equal."""
    return values.sort(dim=-1, descending=True, stable=True).indices


def _plain_route(case, s):
    x, keep = s["x"].float(), s["keep"] != 0
    T, E = x.shape
    K, groups, top_groups = case["K"], case["groups"], case["top_groups"]
    if s["bias"] is None and (groups == 1 or case["group_top"] == 1):
        value = x                                                       # scores rise with the logits
    else:                                                               # 64 bits: borders between scores
        value = torch.where(x == float("-inf"), float("-inf"), _scores(x.double(), case["scores"]))
        if s["bias"] is not None:
            value = value + s["bias"].double()
    if groups > 1:
        of_group = value.view(T, groups, E // groups).sort(dim=2, descending=True).values[:, :, :case["group_top"]]
        none = of_group[:, :, 0] == float("-inf")
        total = torch.where(of_group == float("-inf"), 0.0, of_group).sum(2)
        first = _descending(torch.where(none, float("-inf"), total))[:, :top_groups]
        inside = torch.zeros(T, groups, dtype=torch.bool, device=x.device).scatter_(1, first, True)
        value = torch.where(inside.repeat_interleave(E // groups, 1), value, float("-inf"))
    chosen = _descending(value)[:, :K]
    there = (value.gather(1, chosen) > float("-inf")) & keep[:, None]
    weight = torch.where(there, _scores(x, case["scores"]).gather(1, chosen), 0.0)
    if case["renormalise"]:
        total = weight.sum(1, keepdim=True)
        weight = weight / torch.where(total == 0, 1.0, total)
    return {"chosen": torch.where(there, chosen, -1).to(torch.int32), "weight": weight * case["scale"]}


def _plain_route_gradient(case, s):
    x, keep = s["x"].float(), s["keep"] != 0
    chosen = s["chosen"].long()
    there = (chosen >= 0) & keep[:, None]
    at = chosen.clamp(min=0)
    dw = torch.where(there, s["dweight"], 0.0) * case["scale"]
    score = _scores(x, case["scores"])
    picked = torch.where(there, score.gather(1, at), 0.0)
    if case["renormalise"]:                                             # weight = picked / total
        total = picked.sum(1, keepdim=True)
        total = torch.where(total == 0, 1.0, total)
        dw = torch.where(there, (dw - (dw * picked).sum(1, keepdim=True) / total) / total, 0.0)
    d_score = torch.zeros_like(x).scatter_add_(1, at, dw)
    if case["scores"] == "softmax":
        dx = score * (d_score - (d_score * score).sum(1, keepdim=True))
    else:
        dx = d_score * score * (1.0 - score)
    if s["plus"] is not None:
        dx = dx + s["plus"].float()
    return {"dx": dx.to(s["x"].dtype)}


def _plain_product(s):
    x, w, chosen = s["x"], s["w"], s["chosen"].reshape(-1)
    K = s["chosen"].shape[1]
    y = torch.zeros(chosen.numel(), w.shape[1], device=x.device)
    for e in range(w.shape[0]):
        rows = (chosen == e).nonzero().squeeze(1)
        of = x.reshape(-1, x.shape[-1])[rows] if x.dim() == 3 else x[rows // K]
        y[rows] = of.float() @ w[e].float().t()
    return {"y": y.to(x.dtype).view(*s["chosen"].shape, -1)}


def _plain_product_gradient(s):
    x, w, chosen = s["x"], s["w"], s["chosen"].reshape(-1)
    K = s["chosen"].shape[1]
    dy = s["dy"].reshape(chosen.numel(), -1)
    dx = torch.zeros(chosen.numel(), x.shape[-1], device=x.device)
    dw = torch.zeros(w.shape, device=x.device)
    for e in range(w.shape[0]):
        rows = (chosen == e).nonzero().squeeze(1)
        of = x.reshape(-1, x.shape[-1])[rows] if x.dim() == 3 else x[rows // K]
        d = dy[rows].float()
        dx[rows] = d @ w[e].float()
        dw[e] = d.t() @ of.float()
    dx = dx.view(*s["chosen"].shape, -1)
    return {"dx": (dx if x.dim() == 3 else dx.sum(1)).to(x.dtype), "dw": dw}


def _plain_clip(case, s):
    norms = []
    for g, out in zip(s["g"], s["out"]):
        square = torch.zeros((), dtype=torch.float64, device=g.device)          # 64 bits: long sums
        for at, n in s["rows"]:
            square = square + g[at:at + n].square().sum(dtype=torch.float64)
        norm = square.sqrt() * abs(case["scale"])
        by = (s["max_norm"] / norm).clamp(max=1.0) * case["scale"]
        for at, n in s["rows"]:
            out[at:at + n] = g[at:at + n] * by.float()
        norms.append(norm.float())
    return {"norm": torch.stack(norms), "out": s["out"]}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    op = case["op"]
    if op == "clip":
        n = case["W"] * sum(map(int, case["sizes"].split()))
        return {"bytes": 8 * n + 4 * case["W"], "flops": 3 * n}
    size = 4 if case["type"] == "f32" else 2
    T, E, K = case["T"], case["E"], case["K"]
    if op == "route":
        return {"bytes": T * E * size + 8 * T * K + T + (4 * E if case["bias"] else 0), "flops": T * E * (6 + 2 * K)}
    if op == "route_gradient":
        dense = case["scores"] == "softmax" and not case["renormalise"]         # else only the chosen logits matter
        read = (T * E if dense else T * K) + (T * E if case["plus"] else 0)
        return {"bytes": (read + T * E) * size + 8 * T * K + T, "flops": T * E * (8 if dense else 1) + 10 * T * K}
    D, F = case["in"], case["out"]
    n = T * K * (1.0 - case["nobody"])
    used = E * (1.0 - (1.0 - 1.0 / E) ** n)                                     # experts that have a row
    x = T * D * (K if case["per_slot"] else 1) * size
    rows = T * K * F * size
    if op == "product":
        return {"bytes": int(x + used * D * F * size + rows) + 4 * T * K, "flops": int(2 * n * D * F)}
    return {"bytes": int(2 * x + used * D * F * size + rows) + 4 * E * D * F + 4 * T * K, "flops": int(4 * n * D * F)}


# ------------------------------------------------------------------ the definition, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"route": _exact_route, "route_gradient": _exact_route_gradient, "product": _exact_product,
            "product_gradient": _exact_product_gradient, "clip": _exact_clip}[case["op"]](case, s)


def _log_scores(x, scores):
    return torch.log_softmax(x, 1) if scores == "softmax" else -torch.logaddexp(torch.zeros_like(x), -x)


def _exact_route(case, s):
    """One slot after the other: the best expert that is left.  Weights from the scores' logarithms."""
    x = s["x"].double()
    T, E = x.shape
    K, G = case["K"], case["groups"]
    dead = x == float("-inf")
    log_score = _log_scores(torch.where(dead.all(1, keepdim=True), 0.0, x), case["scores"])
    log_score = torch.where(dead, float("-inf"), log_score)
    c = log_score.exp() if s["bias"] is None else log_score.exp() + s["bias"].double()
    if s["bias"] is None and (G == 1 or case["group_top"] == 1):
        c = x
    expert = torch.arange(E, device=DEVICE)
    open_ = ~dead & (s["keep"] != 0)[:, None]

    def best(values, allowed):
        """The largest allowed value's lowest position, and whether there is one."""
        v = torch.where(allowed, values, float("-inf"))
        top = v.max(1, keepdim=True).values
        where = torch.where(allowed & (v == top), torch.arange(v.shape[1], device=DEVICE), v.shape[1]).min(1).values
        return where, where < v.shape[1]

    if G > 1:
        group_value = torch.zeros(T, G, dtype=torch.float64, device=DEVICE)
        left = open_.clone()
        for _ in range(case["group_top"]):
            for g in range(G):
                part = slice(g * (E // G), (g + 1) * (E // G))
                at, found = best(c[:, part], left[:, part])
                at = at.clamp(max=E // G - 1) + g * (E // G)
                group_value[:, g] += torch.where(found, c[torch.arange(T, device=DEVICE), at], 0.0)
                left[torch.arange(T, device=DEVICE)[found], at[found]] = False
        allowed = open_.view(T, G, E // G).any(2)
        taken = torch.zeros(T, G, dtype=torch.bool, device=DEVICE)
        for _ in range(case["top_groups"]):
            at, found = best(group_value, allowed & ~taken)
            taken[torch.arange(T, device=DEVICE)[found], at[found]] = True
        open_ = open_ & taken[:, expert // (E // G)]
    chosen = torch.full((T, K), -1, dtype=torch.int32, device=DEVICE)
    logs = torch.full((T, K), float("-inf"), dtype=torch.float64, device=DEVICE)
    for k in range(K):
        at, found = best(c, open_)
        r = torch.arange(T, device=DEVICE)[found]
        chosen[r, k] = at[found].to(torch.int32)
        logs[r, k] = log_score[r, at[found]]
        open_[r, at[found]] = False
    if case["renormalise"]:
        total = torch.logsumexp(logs, 1, keepdim=True)
        logs = logs - torch.where(total == float("-inf"), 0.0, total)
    return {"chosen": chosen, "weight": case["scale"] * logs.exp()}


def _exact_route_gradient(case, s):
    """Through the weights' logarithms: d log score_k / d x_j is [k = j] - p_j for a softmax, [k = j] (1 - s_j) for a sigmoid."""
    x = s["x"].double()
    E = x.shape[1]
    log_score = _log_scores(x, case["scores"])
    there = (s["chosen"] >= 0) & (s["keep"] != 0)[:, None]
    pick = torch.nn.functional.one_hot(s["chosen"].long().clamp(min=0), E)
    dx = torch.zeros_like(x)
    for i in torch.arange(x.shape[0], device=DEVICE).split(16384):
        hot = pick[i].double() * there[i, :, None]
        logs = torch.where(there[i], log_score[i].gather(1, s["chosen"][i].long().clamp(min=0)), float("-inf"))
        if case["renormalise"]:
            total = torch.logsumexp(logs, 1, keepdim=True)
            logs = logs - torch.where(total == float("-inf"), 0.0, total)
        by_log = torch.where(there[i], s["dweight"][i].double(), 0.0) * case["scale"] * logs.exp()
        if case["renormalise"]:
            by_log = by_log - logs.exp() * by_log.sum(1, keepdim=True)
        by_expert = (hot * by_log[:, :, None]).sum(1)
        p = log_score[i].exp()
        if case["scores"] == "softmax":
            dx[i] = by_expert - p * by_log.sum(1, keepdim=True) * (0.0 if case["renormalise"] else 1.0)
        else:
            dx[i] = by_expert * (-torch.expm1(log_score[i]))
    return {"dx": dx if s["plus"] is None else dx + s["plus"].double()}


def _by_expert(s):
    """The rows (token * K + slot) of every expert that has any, from one sort."""
    flat = s["chosen"].reshape(-1).long()
    rows = flat.argsort(stable=True)
    for e, n in zip(*(t.tolist() for t in flat.unique(return_counts=True))):
        mine, rows = rows[:n], rows[n:]
        if e >= 0:
            yield e, mine


def _exact_product(case, s):
    x = (s["x"] if case["per_slot"] else s["x"][:, None].expand(-1, case["K"], -1)).reshape(-1, case["in"])
    y = torch.zeros(case["T"] * case["K"], case["out"], dtype=torch.float64, device=DEVICE)
    for e, rows in _by_expert(s):
        y[rows] = torch.mm(x[rows].double(), s["w"][e].double().t())
    return {"y": y.view(case["T"], case["K"], -1)}


def _exact_product_gradient(case, s):
    T, K, D = case["T"], case["K"], case["in"]
    dx = torch.zeros(s["x"].shape, dtype=torch.float64, device=DEVICE).view(-1, D)
    dw = torch.zeros(s["w"].shape, dtype=torch.float64, device=DEVICE)
    x, dy = s["x"].view(-1, D), s["dy"].view(T * K, -1)
    for e, rows in _by_expert(s):
        d = dy[rows].double()
        source = rows if case["per_slot"] else rows // K
        dx.index_add_(0, source, torch.mm(d, s["w"][e].double()))
        dw[e] = torch.mm(d.t(), x[source].double())
    return {"dx": dx.view(s["x"].shape), "dw": dw}


def _exact_clip(case, s):
    norms, outs = [], []
    inside = torch.zeros(s["g"][0].shape, dtype=torch.bool, device=DEVICE)
    for at, n in s["rows"]:
        inside[at:at + n] = True
    for g in s["g"]:
        scaled = torch.where(inside, g.double() * case["scale"], 0.0)
        norm = torch.linalg.vector_norm(scaled)
        outs.append(scaled * torch.clamp(s["max_norm"] / norm, max=1.0))
        norms.append(norm)
    return {"norm": torch.stack(norms), "out": outs}
