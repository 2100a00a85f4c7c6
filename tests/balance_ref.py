"""The balance losses and their gradient in 64 bits, from the formulas: what the kernels are compared with."""
import numpy as np


def sequences(T, seq_offsets, token_mask):
    """Indices of each sequence's tokens that take part."""
    off = [0, T] if seq_offsets is None else [int(v) for v in seq_offsets]
    on = np.ones(T, bool) if token_mask is None else np.asarray(token_mask) != 0
    return [np.array([t for t in range(a, b) if on[t]], dtype=np.int64) for a, b in zip(off[:-1], off[1:])]


def rows(logits, sigmoid):
    """probabilities, softmax, sigmoids, logsumexp; a row without a finite logit has none"""
    l = np.asarray(logits, np.float64)
    T, E = l.shape
    p, soft, sig, lse = np.zeros((T, E)), np.zeros((T, E)), np.zeros((T, E)), np.zeros(T)
    for t in range(T):
        m = l[t].max()
        if m == -np.inf:
            continue
        ex = np.exp(l[t] - m)
        soft[t], lse[t] = ex / ex.sum(), m + np.log(ex.sum())
        with np.errstate(over="ignore"):
            sig[t] = 1.0 / (1.0 + np.exp(-l[t]))
        p[t] = soft[t]
        if sigmoid:   # exp(l) / (1 + exp(l)), scaled by the largest where that is small
            n = np.exp(l[t] - min(m, 0.0)) / (1.0 + np.exp(l[t])) if m < 0 else sig[t]
            p[t] = n / n.sum()
    return p, soft, sig, lse


def fwd(logits, ids, seq_offsets=None, token_mask=None, sigmoid=False):
    T, E = np.asarray(logits).shape
    ids = np.asarray(ids)
    k = ids.shape[1]
    seqs = sequences(T, seq_offsets, token_mask)
    p, _, _, lse = rows(logits, sigmoid)
    n = len(seqs)
    counts, prob, tokens = np.zeros((n, E), np.int32), np.zeros((n, E)), np.zeros(n + 1, np.int32)
    balance = 0.0
    for s, ts in enumerate(seqs):
        tokens[s] = len(ts)
        for t in ts:
            for e in ids[t]:
                if 0 <= e < E:
                    counts[s, e] += 1
        if len(ts):
            prob[s] = p[ts].mean(0)
            balance += E / (k * len(ts)) * (counts[s] * prob[s]).sum() / n
    tokens[n] = tokens[:n].sum()
    z = sum((lse[ts] ** 2).sum() for ts in seqs) / max(int(tokens[n]), 1)
    return np.array([balance, z]), counts, prob, tokens


def bwd(logits, ids, counts, tokens, d_losses, d_topk_w=None, seq_offsets=None, token_mask=None, sigmoid=False, renorm=False):
    """-> gradient, and for every row the size of what is added up in it (for tolerances)"""
    T, E = np.asarray(logits).shape
    p, soft, sig, lse = rows(logits, sigmoid)
    d, size = np.zeros((T, E)), np.zeros(T)
    seqs = sequences(T, seq_offsets, token_mask)
    n = len(seqs)
    for s, ts in enumerate(seqs):
        for t in ts:
            k = ids.shape[1]
            x = d_losses[0] * E / (k * n) / float(tokens[s]) ** 2 * counts[s]
            d[t] += p[t] * (x - (p[t] * x).sum()) * ((1 - sig[t]) if sigmoid else 1.0)
            zc = 2 * d_losses[1] * lse[t] / tokens[n]
            d[t] += zc * soft[t]
            size[t] += abs(x).max() + abs(zc)
    if d_topk_w is not None:
        v = sig if sigmoid else soft
        for t in range(T):
            named = [(int(e), float(g)) for e, g in zip(ids[t], d_topk_w[t]) if 0 <= e < E]
            size[t] += sum(abs(g) for _, g in named)
            if renorm:
                Z = sum(v[t, e] for e, _ in named)
                if Z == 0:
                    continue
                dot = sum(g * v[t, e] / Z for e, g in named)
                for e, g in named:
                    d[t, e] += v[t, e] / Z * (g - dot) * ((1 - v[t, e]) if sigmoid else 1.0)
            elif sigmoid:
                for e, g in named:
                    d[t, e] += g * v[t, e] * (1 - v[t, e])
            else:
                x = np.zeros(E)
                for e, g in named:
                    x[e] += g
                d[t] += soft[t] * (x - (soft[t] * x).sum())
    return d, size
