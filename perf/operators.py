"""Performance cases of the router's balance losses and of the experts with 4-bit weights.

A case is a dict of plain values.  `op` says which operator a pass goes through, the rest are sizes and options:

  balance     a training step's balance and z losses of the router with the per-expert counts of every sequence, then the
              whole gradient of the logits: of both losses and of the routing scores
  experts     the layer's forward with expert weights in 4 bits and a scale (and a zero point, `asym`) per `group` of the reduction
  weights     bf16 weights brought into 4 bits, and the values they stand for (in bf16)

T tokens, d hidden size, E routed experts, k per token, S shared experts, F expert intermediate size; `gate` softmax or sigmoid,
`renorm` the k scores; `seqs` sequences of uneven length in the T tokens, `masked` the share of padding tokens among them;
`n` matrices of `rows` x `cols`.
"""
import math
import random

import torch

own = False   # True: run() makes the framework's calls; False: the operators' plain form

BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32


def listed():
    def balance(name, T, E, k, **more):
        return dict({"name": name, "op": "balance", "T": T, "E": E, "k": k, "gate": "softmax", "renorm": True, "seqs": 1, "masked": 0.0}, **more)

    def experts(name, T, d, E, k, S, F, group, asym):
        return {"name": name, "op": "experts", "T": T, "d": d, "E": E, "k": k, "S": S, "F": F, "group": group, "asym": asym}

    def weights(name, n, rows, cols, group, asym):
        return {"name": name, "op": "weights", "n": n, "rows": rows, "cols": cols, "group": group, "asym": asym}

    return [
        # the smallest training step (workloads/configs.py, configuration 0): launches and host time
        balance("balance_tiny", 256, 8, 2),
        # a training step of the V3-shaped router (configuration 4), eight packed sequences
        balance("balance_8192", 8192, 256, 8, seqs=8),
        # an expert count and a token count that fit no vector or tile; scores not renormalised
        balance("balance_odd", 1777, 130, 6, renorm=False, seqs=3),
        # a large batch of uneven sequences with padding tokens, sigmoid scores: bound by memory
        balance("balance_65536", 65536, 256, 8, gate="sigmoid", seqs=97, masked=0.1),
        # one sequence generates a token, V2-Lite-shaped layer (configuration 1): the smallest serving call
        experts("experts_lite_1", 1, 2048, 64, 6, 2, 1408, 128, False),
        # eight sequences generate, V3-shaped experts, the 32 experts of one rank: bound by the weights
        experts("experts_v3_8", 8, 7168, 32, 8, 1, 2048, 128, False),
        # a serving batch, a few tokens to an expert, zero points and small groups
        experts("experts_lite_64", 64, 2048, 64, 6, 2, 1408, 64, True),
        # a short prompt or a chunk of one: some fifty tokens to an expert
        experts("experts_lite_512", 512, 2048, 64, 6, 2, 1408, 128, False),
        # prompt processing: bound by the products
        experts("experts_lite_4096", 4096, 2048, 64, 6, 2, 1408, 128, False),
        # sizes that fit no tile and no group
        experts("experts_ragged_333", 333, 1160, 24, 3, 1, 712, 32, True),
        # the gate and up projections of a V2-Lite-shaped layer when a checkpoint is loaded
        weights("weights_lite", 64, 2816, 2048, 128, False),
        # ragged matrices with zero points
        weights("weights_ragged", 25, 1160, 712, 32, True),
    ]


# ---------------------------------------------------------------- what a pass cannot do without
def _hit(c):
    """Expected number of routed experts that receive a token."""
    return c["E"] * (1.0 - (1.0 - c["k"] / c["E"]) ** c["T"])


def _bytes_per_weight(c):
    return 0.5 + (2.0 + (1.0 if c["asym"] else 0.0)) / c["group"]


def work(case):
    c = case
    if c["op"] == "balance":   # logits, ids, score gradient -> gradient, counts, mean probabilities
        return {"bytes": 8.0 * c["T"] * c["E"] + 8.0 * c["T"] * c["k"] + 8.0 * c["seqs"] * c["E"], "flops": 0.0}
    if c["op"] == "weights":   # the bf16 matrices in, the values out
        return {"bytes": c["n"] * c["rows"] * c["cols"] * 4.0, "flops": 0.0}
    rows = c["T"] * (c["k"] + c["S"])
    return {"bytes": (_hit(c) + c["S"]) * 3.0 * c["d"] * c["F"] * _bytes_per_weight(c) + 4.0 * c["T"] * c["d"] + 8.0 * c["T"] * c["k"],
            "flops": 6.0 * rows * c["d"] * c["F"]}


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same operators, its sizes spread over the listed ranges; never dearer than the dearest listed case of its operator."""
    op = rng.choice(["balance", "balance", "experts", "experts", "experts", "weights"])
    most = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        if op == "balance":
            E = rng.choice([4, 8, 24, 40, 64, 100, 128, 130, 160, 256, 321, 512])
            c = {"op": op, "T": _log_int(rng, 16, 65536), "E": E, "k": rng.randint(1, min(8, E)), "gate": rng.choice(["softmax", "softmax", "sigmoid"]),
                 "renorm": rng.random() < 0.6, "seqs": 1, "masked": rng.choice([0.0, 0.0, 0.2])}
            c["seqs"] = _log_int(rng, 1, min(256, c["T"]))
        elif op == "experts":
            E = rng.choice([8, 16, 24, 32, 40, 64])
            c = {"op": op, "T": _log_int(rng, 1, 4096), "d": 8 * _log_int(rng, 32, 896), "E": E, "k": rng.randint(1, min(8, E)), "S": rng.choice([0, 0, 1, 2]),
                 "F": 8 * _log_int(rng, 16, 256), "group": rng.choice([32, 64, 128, 128]), "asym": rng.random() < 0.4}
            if 3.0 * (E + c["S"]) * c["d"] * c["F"] > 1.5e9:
                continue
        else:
            c = {"op": op, "n": _log_int(rng, 1, 64), "rows": 16 * _log_int(rng, 8, 256), "cols": 8 * _log_int(rng, 16, 896),
                 "group": rng.choice([32, 64, 128]), "asym": rng.random() < 0.5}
        if _cost(c) <= most:
            return c


# ---------------------------------------------------------------- what a program has in hand
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, shape, std, dtype=BF16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def _inputs_balance(c, seed):
    """Logits as x.W_r gives them (x ~ N(0, 1), W_r ~ N(0, 0.02), d = 7168), their selection, the gradients that arrive."""
    T, E, k = c["T"], c["E"], c["k"]
    gen, rng = _gen(seed), random.Random(seed)
    logits = _normal(gen, (T, E), 1.7, F32)
    ids = torch.topk(logits, k, dim=1).indices.to(I32).contiguous()
    cuts = sorted(rng.randint(0, T) for _ in range(c["seqs"] - 1))
    offsets = torch.tensor([0] + cuts + [T], dtype=I32, device="cuda")
    mask = None
    if c["masked"]:
        mask = (torch.rand(T, generator=gen, device="cuda") >= c["masked"]).to(torch.uint8)
    d_losses = torch.tensor([1e-2, 1e-3], device="cuda")
    return {"logits": logits, "ids": ids, "offsets": offsets, "mask": mask, "d_topk_w": _normal(gen, (T, k), 1e-3, F32), "d_losses": d_losses}


def _inputs_codes(gen, n, rows, cols, group, asym):
    """A checkpoint's natural form: codes two to a byte (the even column in the low half), scales and zero points of each group."""
    groups = -(-cols // group)
    q = torch.randint(0, 256, (n, rows, cols // 2), dtype=torch.uint8, device="cuda", generator=gen)
    # weights of variance 1 / cols: codes are spread evenly over 16 steps, whose variance is (16^2 - 1) / 12
    s = (torch.rand(n, rows, groups, device="cuda", generator=gen) + 0.5).mul_(cols ** -0.5 / 4.6).to(BF16)
    z = torch.randint(6, 10, (n, rows, groups), dtype=torch.uint8, device="cuda", generator=gen) if asym else None
    return q, s, z


def _inputs_experts(c, seed):
    T, d, E, k, S, F = (c[n] for n in ("T", "d", "E", "k", "S", "F"))
    gen = _gen(seed)
    s = {"x": _normal(gen, (T, d), 1.0)}
    score, ids = torch.topk(_normal(gen, (T, E), 1.0, F32), k, dim=1)
    s["ids"], s["w"] = ids.to(I32).contiguous(), torch.softmax(score, 1).contiguous()
    s["gate_up"] = _inputs_codes(gen, E + S, 2 * F, d, c["group"], c["asym"])
    s["down"] = _inputs_codes(gen, E + S, d, F, c["group"], c["asym"])
    return s


def prepare(case, seed):
    c = case
    if c["op"] == "balance":
        s = _inputs_balance(c, seed)
        if own:
            from paper_2605_23764_b200 import MoeLayer
            s["layer"] = MoeLayer(c["T"], 64, c["E"], c["k"], 0, 64, renorm=c["renorm"], sigmoid_gate=c["gate"] == "sigmoid")
    elif c["op"] == "experts":
        s = _inputs_experts(c, seed)
        if own:   # the weights are laid out once, when the checkpoint is loaded
            from paper_2605_23764_b200 import MoeLayer, MoeW4Weights
            s["layer"] = MoeLayer(c["T"], c["d"], c["E"], c["k"], c["S"], c["F"], w4=True)
            s["W_gate_up"] = MoeW4Weights.pack(*s["gate_up"], group=c["group"], gate_up=True)
            s["W_down"] = MoeW4Weights.pack(*s["down"], group=c["group"])
    else:
        s = {"W": _normal(_gen(seed), (c["n"], c["rows"], c["cols"]), c["cols"] ** -0.5)}
    s["c"] = c
    return s


# ---------------------------------------------------------------- the plain forms
def _balance_plain(s):
    c, l = s["c"], s["logits"]
    T, E, k, n = c["T"], c["E"], c["k"], c["seqs"]
    # the sequence of each token; a row of its own for tokens that take no part
    seq = torch.searchsorted(s["offsets"][1:].contiguous(), torch.arange(T, dtype=I32, device="cuda"), right=True)
    if s["mask"] is not None:
        seq = torch.where(s["mask"] != 0, seq, n)
    ids = s["ids"].long()
    m = l.amax(1, keepdim=True)
    ex = torch.exp(l - m)
    soft = ex / ex.sum(1, keepdim=True)
    lse = (m + torch.log(ex.sum(1, keepdim=True))).squeeze(1)
    sig = 1.0 / (1.0 + torch.exp(-l))
    p = sig / sig.sum(1, keepdim=True) if c["gate"] == "sigmoid" else soft
    # per sequence: tokens, slots of each expert, mean probabilities
    tokens = torch.zeros(n + 1, dtype=torch.int64, device="cuda").index_add_(0, seq, torch.ones_like(seq))[:n]
    counts = torch.zeros((n + 1) * E, dtype=torch.int64, device="cuda")
    counts = counts.index_add_(0, (seq[:, None] * E + ids).view(-1), torch.ones(T * k, dtype=torch.int64, device="cuda")).view(n + 1, E)[:n]
    psum = torch.zeros(n + 1, E, dtype=F64, device="cuda").index_add_(0, seq, p.double())[:n]
    ns = tokens.clamp(min=1).double()[:, None]
    prob = psum / ns
    total = tokens.sum()
    live = seq < n
    balance = (E / (k * n) / ns * counts * prob).sum()
    z = torch.where(live, lse.double().square(), 0.0).sum() / total.clamp(min=1)
    # gradients
    coef = (s["d_losses"][0] * (E / (k * n)) / ns.square() * counts).to(F32)
    x = torch.cat([coef, torch.zeros(1, E, device="cuda")])[seq]
    inner = x - (p * x).sum(1, keepdim=True)
    dl = p * inner * (1.0 - sig) if c["gate"] == "sigmoid" else p * inner
    dl = dl + torch.where(live, 2.0 * s["d_losses"][1] / total.clamp(min=1) * lse, 0.0)[:, None] * soft
    g, chosen = s["d_topk_w"], torch.gather(sig if c["gate"] == "sigmoid" else soft, 1, ids)
    if c["renorm"]:
        w = chosen / chosen.sum(1, keepdim=True)
        dsel = w * (g - (g * w).sum(1, keepdim=True))
        dl = dl.scatter_add(1, ids, dsel * (1.0 - chosen) if c["gate"] == "sigmoid" else dsel)
    elif c["gate"] == "sigmoid":
        dl = dl.scatter_add(1, ids, g * chosen * (1.0 - chosen))
    else:
        dl = dl - soft * (g * chosen).sum(1, keepdim=True)
        dl = dl.scatter_add(1, ids, g * chosen)
    return {"losses": torch.stack([balance, z]).to(F32), "counts": counts.to(I32), "prob": prob.to(F32), "d_logits": dl}


def _values(q, s, z, group):
    """The weights that natural codes stand for, in 32 bits."""
    cols = 2 * q.shape[2]
    v = torch.stack([q & 15, q >> 4], 3).view(q.shape[0], q.shape[1], cols).to(F32)
    of = torch.arange(cols, device="cuda") // group
    v -= 8.0 if z is None else z.to(F32)[:, :, of]
    v *= s.to(F32)[:, :, of]
    return v


def _swiglu(x, W1):
    """silu(x Wg^T) * (x Wu^T) for the rows of each expert."""
    h = torch.bmm(x, W1.transpose(1, 2))
    g, u = h.chunk(2, dim=2)
    return g / (1.0 + torch.exp(-g)) * u


def _experts_plain(s):
    c = s["c"]
    T, d, E, k, S = (c[n] for n in ("T", "d", "E", "k", "S"))
    x, ids, w = s["x"].to(F32), s["ids"].long(), s["w"]
    out = torch.zeros(T, d, device="cuda")
    flat = ids.view(-1)
    hit, of, count = torch.unique(flat, return_inverse=True, return_counts=True)
    order = torch.argsort(of, stable=True)
    place = torch.empty_like(of)   # of each slot among the rows of its expert
    place[order] = torch.arange(T * k, device="cuda") - (torch.cumsum(count, 0) - count)[of[order]]
    rows = torch.zeros(len(hit), int(count.max()), d, device="cuda")
    token = torch.arange(T * k, device="cuda") // k
    rows[of, place] = x[token]
    take = lambda part, e: _values(*(None if t is None else t[e] for t in part), c["group"])
    a = _swiglu(rows, take(s["gate_up"], hit))
    y = torch.bmm(a, take(s["down"], hit).transpose(1, 2))
    out.index_add_(0, token, y[of, place] * w.view(-1, 1))
    if S:
        shared = torch.arange(E, E + S, device="cuda")
        a = _swiglu(x.expand(S, T, d), take(s["gate_up"], shared))
        out += torch.bmm(a, take(s["down"], shared).transpose(1, 2)).sum(0)
    return {"out": out.to(BF16)}


def _in_groups(W, group):
    """[n][rows][groups][group], zeros behind the last column."""
    n, rows, cols = W.shape
    pad = -cols % group
    return torch.nn.functional.pad(W.to(F32), (0, pad)).view(n, rows, -1, group)


def _weights_plain(s):
    c, W = s["c"], s["W"]
    v = _in_groups(W, c["group"])
    if c["asym"]:
        lo, hi = v.amin(3, keepdim=True).clamp(max=0.0), v.amax(3, keepdim=True).clamp(min=0.0)
        scale = ((hi - lo) / 15.0).to(BF16).to(F32)
        step = torch.where(scale > 0, scale, 1.0)
        zero = torch.round(-lo / step).clamp(0, 15)
        q = (torch.round(v / step) + zero).clamp(0, 15)
    else:
        scale = (v.abs().amax(3, keepdim=True) / 7.0).to(BF16).to(F32)
        step = torch.where(scale > 0, scale, 1.0)
        zero = 8.0
        q = torch.round(v / step).clamp(-8, 7) + 8.0
    return {"values": (scale * (q - zero)).view(c["n"], c["rows"], -1)[:, :, :c["cols"]].to(BF16).contiguous()}


# ---------------------------------------------------------------- one pass
def run(s):
    c = s["c"]
    if not own:
        return {"balance": _balance_plain, "experts": _experts_plain, "weights": _weights_plain}[c["op"]](s)
    if c["op"] == "balance":
        layer = s["layer"]
        losses, counts, prob, tokens = layer.balance_fwd(s["logits"], s["ids"], s["offsets"], s["mask"])
        d_logits = layer.balance_bwd(s["logits"], s["ids"], counts, tokens, s["d_losses"], s["d_topk_w"], s["offsets"], s["mask"])
        return {"losses": losses, "counts": counts, "prob": prob, "d_logits": d_logits}
    if c["op"] == "experts":
        return {"out": s["layer"].ffn_fwd_w4(s["x"], s["ids"], s["w"], s["W_gate_up"], s["W_down"])}
    from paper_2605_23764_b200 import MoeW4Weights
    return {"values": MoeW4Weights.quantize(s["W"], group=c["group"], asymmetric=c["asym"]).dequantize()}


# ---------------------------------------------------------------- the definitions in 64 bits
def _exact_balance(c, s):
    """Both losses from their definition, sequence by sequence; the gradients by differentiating them and the scores."""
    l = s["logits"].double().requires_grad_()
    T, E, k, n = c["T"], c["E"], c["k"], c["seqs"]
    on = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"] != 0
    scores = torch.sigmoid(l) if c["gate"] == "sigmoid" else torch.softmax(l, 1)
    p = scores / scores.sum(1, keepdim=True)
    balance, counts, prob = 0.0, [], []
    ends = s["offsets"].tolist()
    for a, b in zip(ends[:-1], ends[1:]):
        q, named = p[a:b][on[a:b]], s["ids"][a:b][on[a:b]]
        cnt = torch.bincount(named.reshape(-1).long(), minlength=E)
        mean = q.sum(0) / max(len(q), 1)
        balance = balance + E / k * (cnt / max(len(q), 1) * mean).sum() / n
        counts.append(cnt)
        prob.append(mean.detach())
    z = torch.logsumexp(l[on], 1).square().mean() if bool(on.any()) else l.sum() * 0.0
    w = torch.gather(scores, 1, s["ids"].long())
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    g = s["d_losses"].double()
    (g[0] * balance + g[1] * z + (w * s["d_topk_w"].double()).sum()).backward()
    return {"losses": torch.stack([balance.detach(), z.detach()]), "counts": torch.stack(counts).to(I32), "prob": torch.stack(prob), "d_logits": l.grad}


def _exact_matrix(part, e, group):
    q, s, z = (None if t is None else t[e] for t in part)
    codes = torch.empty(q.shape[0], 2 * q.shape[1], dtype=F64, device="cuda")
    codes[:, 0::2], codes[:, 1::2] = (q % 16).double(), torch.div(q, 16, rounding_mode="floor").double()
    zero = torch.full(s.shape, 8.0, dtype=F64, device="cuda") if z is None else z.double()
    spread = lambda t: t.repeat_interleave(group, 1)[:, :codes.shape[1]]
    return (codes - spread(zero)) * spread(s.double())


def _exact_experts(c, s):
    T, d, E, F = c["T"], c["d"], c["E"], c["F"]
    x, out = s["x"].double(), torch.zeros(T, d, dtype=F64, device="cuda")
    for e in range(E + c["S"]):
        if e < E:
            t, j = torch.nonzero(s["ids"] == e, as_tuple=True)
            w = s["w"][t, j].double()
        else:
            t, w = torch.arange(T, device="cuda"), torch.ones(T, dtype=F64, device="cuda")
        if not len(t):
            continue
        h = x[t] @ _exact_matrix(s["gate_up"], e, c["group"]).T
        a = torch.nn.functional.silu(h[:, :F]) * h[:, F:]
        out.index_add_(0, t, w[:, None] * (a @ _exact_matrix(s["down"], e, c["group"]).T))
    return {"out": out}


def _exact_weights(c, s):
    out = torch.empty(s["W"].shape, dtype=F64, device="cuda")
    bf = lambda t: t.to(F32).to(BF16).double()   # scales are held in bf16, by definition
    for a in range(0, c["cols"], c["group"]):
        v = s["W"][:, :, a:a + c["group"]].double()
        if c["asym"]:
            lo, hi = v.amin(2, keepdim=True).clamp(max=0), v.amax(2, keepdim=True).clamp(min=0)
            scale = bf((hi - lo) / 15)
            zero = torch.nan_to_num(torch.round(-lo / scale)).clamp(0, 15)
            out[:, :, a:a + c["group"]] = scale * ((torch.nan_to_num(torch.round(v / scale)) + zero).clamp(0, 15) - zero)
        else:
            scale = bf(v.abs().amax(2, keepdim=True) / 7)
            out[:, :, a:a + c["group"]] = scale * torch.nan_to_num(torch.round(v / scale)).clamp(-8, 7)
    return {"values": out}


def exact(case, seed):
    c = case
    if c["op"] == "balance":
        return _exact_balance(c, _inputs_balance(c, seed))
    if c["op"] == "experts":
        return _exact_experts(c, _inputs_experts(c, seed))
    return _exact_weights(c, {"W": _normal(_gen(seed), (c["n"], c["rows"], c["cols"]), c["cols"] ** -0.5)})
