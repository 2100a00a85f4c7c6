"""Performance cases of routing by groups with a bias for balance, and of the experts' update by orthogonalised momentum.

A case is a dict of plain values.  `op` says which operator a pass goes through, the rest are sizes and options:

  route   scores of T tokens over E experts in `groups` groups: the `top_groups` best groups by the sum of their `group_top` largest
          biased scores, the k largest biased scores among them, the scores themselves as weights times `scale`; with `train` the
          counts of every expert, the gradient of the logits and the bias of the next step too
  muon    a step of momentum over n weight matrices of rows x cols, orthogonalised, with the weights' update
  ortho   the orthogonalisation by itself, of gradients in bf16 or fp32

`gate` softmax or sigmoid, `renorm` the k weights.  Steps of the orthogonalisation: `steps`.
"""
import math
import random

import torch

own = False   # True: run() makes the framework's calls; False: the operators' plain form

BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
MOMENTUM, LR, DECAY = 0.95, 2e-3, 0.1
BIAS_RATE = 1e-3


def listed():
    def route(name, T, E, k, groups, top_groups, **more):
        return dict({"name": name, "op": "route", "T": T, "E": E, "k": k, "groups": groups, "top_groups": top_groups, "group_top": 2, "gate": "sigmoid",
                     "renorm": True, "scale": 2.5, "bias": True, "train": True}, **more)

    def muon(name, n, rows, cols):
        return {"name": name, "op": "muon", "n": n, "rows": rows, "cols": cols, "steps": 5}

    def ortho(name, n, rows, cols, dtype="bf16", steps=5):
        return {"name": name, "op": "ortho", "n": n, "rows": rows, "cols": cols, "steps": steps, "dtype": dtype}

    return [
        # one sequence generates a token, V3-shaped router (workloads/configs.py, configuration 2): the smallest serving call
        route("route_v3_1", 1, 256, 8, 8, 4, train=False),
        # a training step of the same router (configuration 4)
        route("route_v3_8192", 8192, 256, 8, 8, 4),
        # groups by their best expert, softmax scores as they are, no bias; a group that fits no vector, an odd number of tokens
        route("route_odd_1777", 1777, 150, 6, 10, 3, group_top=1, gate="softmax", renorm=False, scale=16.0, bias=False),
        # a large batch: bound by memory
        route("route_v3_65536", 65536, 256, 8, 8, 4),
        # many experts, softmax scores with a bias, prompt processing (no training)
        route("route_512_16384", 16384, 512, 10, 1, 1, gate="softmax", scale=1.0, train=False),
        # gate and up matrices of the smallest training step (configuration 0): launches and latencies
        muon("muon_tiny", 16, 128, 256),
        # gate and up matrices of the V2-Lite-shaped layer (configuration 1), 66 experts: bound by the products
        muon("muon_lite_gate_up", 132, 1408, 2048),
        # the down matrices of half of its experts: taller than wide
        muon("muon_lite_down", 33, 2048, 1408),
        # the gate matrices of a few V3-shaped experts: wide
        ortho("ortho_v3", 12, 2048, 7168),
        # a router's weights, accumulated in fp32: one matrix, one tile high
        ortho("ortho_router", 1, 256, 7168, "fp32"),
        # sizes that fit no tile and no vector
        ortho("ortho_ragged", 7, 333, 1171),
    ]


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    if c["op"] == "route":
        b = 4.0 * c["T"] * c["E"] + 8.0 * c["T"] * c["k"]            # logits -> ids, weights
        if c["train"]:
            b += 4.0 * c["T"] * c["E"] + 4.0 * c["T"] * c["k"]       # their gradients -> the logits'
        return {"bytes": b, "flops": 0.0}
    m, l = sorted((c["rows"], c["cols"]))
    # X X^T and A A are symmetric: half of their products
    flops = c["n"] * c["steps"] * (m * m * l + m ** 3 + 2.0 * m * m * l)
    each = 14.0 if c["op"] == "muon" else 6.0 if c["dtype"] == "fp32" else 4.0
    return {"bytes": each * c["n"] * c["rows"] * c["cols"], "flops": float(flops)}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    """A case of the same operators, its sizes spread over the listed ranges; never dearer than the dearest listed case of its operator."""
    op = rng.choice(["route", "route", "muon", "ortho"])
    most = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        if op == "route":
            E = rng.choice([8, 16, 24, 40, 64, 96, 128, 150, 160, 192, 256, 384, 512])
            groups = rng.choice([g for g in (1, 2, 3, 4, 5, 8, 10, 16, 32) if E % g == 0 and E // g >= 2])
            top = rng.randint(1, groups)
            c = {"op": op, "T": _log_int(rng, 1, 65536), "E": E, "k": rng.randint(1, min(12, top * (E // groups))), "groups": groups, "top_groups": top,
                 "group_top": rng.choice([1, 2, 2]), "gate": rng.choice(["softmax", "sigmoid", "sigmoid"]), "renorm": rng.random() < 0.6,
                 "scale": rng.choice([1.0, 2.5]), "bias": rng.random() < 0.7, "train": rng.random() < 0.6}
            c["renorm"] &= c["k"] > 1   # one renormalised weight is 1, and has no gradient
        elif op == "muon":
            c = {"op": op, "n": _log_int(rng, 1, 132), "rows": 8 * _log_int(rng, 4, 352), "cols": 8 * _log_int(rng, 4, 896), "steps": 5}
        else:
            c = {"op": op, "n": _log_int(rng, 1, 32), "rows": _log_int(rng, 16, 2816), "cols": _log_int(rng, 16, 7168), "steps": rng.choice([3, 5, 5, 6]),
                 "dtype": rng.choice(["bf16", "bf16", "fp32"])}
        if _cost(c) <= most:
            return c


# ---------------------------------------------------------------- what a program has in hand
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, shape, std, dtype=F32):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def _inputs_route(c, seed):
    """Logits as x.W_r gives them (x ~ N(0, 1), W_r ~ N(0, 0.02), d = 7168), a bias that some hundred steps have moved."""
    gen = _gen(seed)
    s = {"logits": _normal(gen, (c["T"], c["E"]), 1.7), "bias": None}
    if c["bias"]:
        s["bias"] = torch.randint(-100, 101, (c["E"],), generator=gen, device="cuda").to(F32) * BIAS_RATE * (1.0 if c["gate"] == "sigmoid" else 0.05)
    s["d_topk_w"] = _normal(gen, (c["T"], c["k"]), 1e-3)
    return s


def _gradients(gen, n, rows, cols, dtype):
    """Products of activations and their gradients: a spectrum that falls by its index to the power of 0.5, over noise of the
    later tokens; one matrix in sixteen belongs to an expert that received no token."""
    r = min(rows, cols, 512)
    left = _normal(gen, (n, rows, r), 1.0, BF16) * torch.arange(1, r + 1, device="cuda").to(BF16).rsqrt()
    g = torch.baddbmm(_normal(gen, (n, rows, cols), 0.5, BF16), left, _normal(gen, (n, r, cols), 1.0, BF16)).to(dtype).mul_(1e-4)
    g[15::16] = 0
    return g


def _inputs_matrices(c, seed):
    gen = _gen(seed)
    n, rows, cols = c["n"], c["rows"], c["cols"]
    if c["op"] == "ortho":
        return {"G": _gradients(gen, n, rows, cols, F32 if c["dtype"] == "fp32" else BF16)}
    s = {"dW": _gradients(gen, n, rows, cols, BF16)}
    s["M"] = _gradients(gen, n, rows, cols, F32).mul_(8.0)
    s["W"] = _normal(gen, (n, rows, cols), cols ** -0.5, BF16)
    return s


def _adjust(c):
    """Update of the size that a scalar optimiser's has: root mean square 0.2."""
    return 0.2 * math.sqrt(max(c["rows"], c["cols"]))


def prepare(case, seed):
    c = case
    if c["op"] == "route":
        s = _inputs_route(c, seed)
        if own:
            from paper_2605_23764_b200 import MoeLayer
            s["layer"] = MoeLayer(c["T"], 64, c["E"], c["k"], 0, 64, renorm=c["renorm"], sigmoid_gate=c["gate"] == "sigmoid")
    else:
        s = _inputs_matrices(c, seed)
        if own:   # the optimiser with its workspace is made once
            from paper_2605_23764_b200 import MoeMuon
            s["muon"] = MoeMuon(c["n"], c["rows"], c["cols"], momentum=MOMENTUM, coefficients=COEFFICIENTS, steps=c["steps"], eps=EPS)
    s["c"] = c
    return s


# ---------------------------------------------------------------- the plain forms
def _route_plain(s):
    c, l = s["c"], s["logits"]
    T, E, k, G = c["T"], c["E"], c["k"], c["groups"]
    sigmoid = c["gate"] == "sigmoid"
    # which experts: in 64 bits, since scores lie next to one another
    d = l.double()
    if sigmoid:
        choice = 1.0 / (1.0 + torch.exp(-d))
    else:
        ex = torch.exp(d - d.amax(1, keepdim=True))
        choice = ex / ex.sum(1, keepdim=True)
    if s["bias"] is not None:
        choice = choice + s["bias"].double()
    if c["top_groups"] < G:
        best = torch.sort(choice.view(T, G, E // G), dim=2, descending=True).values[:, :, :c["group_top"]].sum(2)
        kept = torch.sort(best, dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        on = torch.zeros(T, G, dtype=torch.bool, device="cuda").scatter_(1, kept, True)
        choice = torch.where(on.repeat_interleave(E // G, dim=1), choice, -math.inf)
    ids = torch.sort(choice, dim=1, descending=True, stable=True).indices[:, :k]
    # their weights
    if sigmoid:
        score = 1.0 / (1.0 + torch.exp(-l))
    else:
        ex = torch.exp(l - l.amax(1, keepdim=True))
        score = ex / ex.sum(1, keepdim=True)
    p = torch.gather(score, 1, ids)
    w = p / p.sum(1, keepdim=True) if c["renorm"] else p
    out = {"ids": ids.to(I32), "w": w * c["scale"]}
    if not c["train"]:
        return out
    counts = torch.zeros(E, dtype=torch.int64, device="cuda").index_add_(0, ids.reshape(-1), torch.ones(T * k, dtype=torch.int64, device="cuda"))
    out["counts"] = counts.to(I32)
    if s["bias"] is not None:
        out["bias"] = s["bias"] + BIAS_RATE * torch.sign(T * k - E * counts).to(F32)
    g = s["d_topk_w"] * c["scale"]
    if c["renorm"]:   # w = p / sum p
        g = (g - (g * w).sum(1, keepdim=True)) / p.sum(1, keepdim=True)
    dl = torch.zeros_like(l)
    if sigmoid:
        out["d_logits"] = dl.scatter_(1, ids, g * p * (1.0 - p))
    else:
        out["d_logits"] = (dl if c["renorm"] else dl - score * (g * p).sum(1, keepdim=True)).scatter_add_(1, ids, g * p)
    return out


def _orthogonal(u, steps):
    """u -> the odd polynomial of its singular values, `steps` times."""
    a, b, c = COEFFICIENTS
    x = u.transpose(1, 2) if u.shape[1] > u.shape[2] else u
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    for _ in range(steps):
        A = torch.bmm(x, x.transpose(1, 2))
        B = b * A + c * torch.bmm(A, A)
        x = a * x + torch.bmm(B, x)
    return x.transpose(1, 2) if u.shape[1] > u.shape[2] else x


def _ortho_plain(s):
    return {"out": _orthogonal(s["G"].to(F32), s["c"]["steps"]).to(BF16).contiguous()}


def _muon_plain(s):
    c, g = s["c"], s["dW"].to(F32)
    M = MOMENTUM * s["M"] + g
    o = _orthogonal(MOMENTUM * M + g, c["steps"])
    W = (1.0 - LR * DECAY) * s["W"].to(F32) - LR * _adjust(c) * o
    return {"W": W.to(BF16).contiguous(), "M": M}


# ---------------------------------------------------------------- one pass
def run(s):
    c = s["c"]
    if not own:
        return {"route": _route_plain, "muon": _muon_plain, "ortho": _ortho_plain}[c["op"]](s)
    if c["op"] == "route":
        layer = s["layer"]
        how = dict(n_groups=c["groups"], top_groups=c["top_groups"], group_top=c["group_top"], scale=c["scale"])
        if not c["train"]:
            ids, w = layer.route_grouped(s["logits"], s["bias"], **how)
            return {"ids": ids, "w": w}
        ids, w, counts = layer.route_grouped(s["logits"], s["bias"], with_counts=True, **how)
        out = {"ids": ids, "w": w, "counts": counts}
        if s["bias"] is not None:
            out["bias"] = layer.bias_update(s["bias"], counts, BIAS_RATE, out=torch.empty_like(s["bias"]))
        out["d_logits"] = layer.route_grouped_bwd(s["logits"], ids, s["d_topk_w"], scale=c["scale"])
        return out
    if c["op"] == "ortho":
        return {"out": s["muon"].orthogonalize(s["G"])}
    W, M = s["muon"].step(s["W"], s["M"], s["dW"], lr=LR, weight_decay=DECAY, scale=_adjust(c), W_out=torch.empty_like(s["W"]), M_out=torch.empty_like(s["M"]))
    return {"W": W, "M": M}


# ---------------------------------------------------------------- the definitions in 64 bits
def _exact_route(c, s):
    """Experts by their rank among all, gradients by differentiating the weights."""
    T, E, k, G = c["T"], c["E"], c["k"], c["groups"]
    l = s["logits"].double().requires_grad_()
    score = torch.sigmoid(l) if c["gate"] == "sigmoid" else torch.softmax(l, 1)
    choice = score.detach().clone()
    if s["bias"] is not None:
        choice += s["bias"].double()
    groups = torch.topk(choice.reshape(T, G, -1), c["group_top"], dim=2).values.sum(2)
    below = torch.arange(G, device="cuda")
    # groups in front of each: larger ones, and equal ones with a lower number
    ahead = ((groups[:, None, :] > groups[:, :, None]) | ((groups[:, None, :] == groups[:, :, None]) & (below[None, None, :] < below[None, :, None]))).sum(2)
    choice[(ahead >= c["top_groups"]).repeat_interleave(E // G, 1)] = -math.inf
    picked, rest = [], choice
    for _ in range(k):
        best = rest.amax(1, keepdim=True)
        one = (rest == best).int().argmax(1, keepdim=True)   # the first of them
        picked.append(one)
        rest = rest.scatter(1, one, -math.inf)
    ids = torch.cat(picked, 1)
    w = torch.gather(score, 1, ids)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    w = w * c["scale"]
    out = {"ids": ids.to(I32), "w": w.detach()}
    if c["train"]:
        counts = torch.bincount(ids.reshape(-1), minlength=E)
        out["counts"] = counts.to(I32)
        if s["bias"] is not None:
            out["bias"] = s["bias"].double() + BIAS_RATE * torch.sign(T * k / E - counts.double())
        (w * s["d_topk_w"].double()).sum().backward()
        out["d_logits"] = l.grad
    return out


def _exact_polar(u, steps):
    """One matrix: the polynomial as products with the smaller Gram matrix."""
    a, b, c = COEFFICIENTS
    u = u / (torch.linalg.norm(u) + EPS)
    for _ in range(steps):
        if u.shape[0] <= u.shape[1]:
            gram = u @ u.T
            u = a * u + b * (gram @ u) + c * (gram @ (gram @ u))
        else:
            gram = u.T @ u
            u = a * u + b * (u @ gram) + c * ((u @ gram) @ gram)
    return u


def exact(case, seed):
    c = case
    if c["op"] == "route":
        return _exact_route(c, _inputs_route(c, seed))
    s = _inputs_matrices(c, seed)
    if c["op"] == "ortho":
        return {"out": torch.stack([_exact_polar(g.double(), c["steps"]) for g in s["G"]])}
    M = MOMENTUM * s["M"].double() + s["dW"].double()
    W = torch.empty(s["W"].shape, dtype=F64, device="cuda")
    for i in range(c["n"]):
        W[i] = (1.0 - LR * DECAY) * s["W"][i].double() - LR * _adjust(c) * _exact_polar(MOMENTUM * M[i] + s["dW"][i].double(), c["steps"])
    return {"W": W, "M": M}
