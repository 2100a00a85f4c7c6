"""Routing by groups with a bias, in 64 bits on the CPU, written as the header states it."""
import numpy as np


def scores(logits, sigmoid):
    l = np.asarray(logits, np.float64)
    if sigmoid:
        with np.errstate(over="ignore"):
            return 1.0 / (1.0 + np.exp(-l))
    m = l.max(1, keepdims=True)
    m = np.where(np.isfinite(m), m, 0.0)
    ex = np.exp(l - m)
    z = ex.sum(1, keepdims=True)
    return np.divide(ex, z, out=np.zeros_like(ex), where=z > 0)


def _order(v):   # indices of falling values, equal ones by index
    return np.lexsort((np.arange(len(v)), -v))


def fwd(logits, k, bias=None, n_groups=1, top_groups=1, group_top=1, scale=1.0, sigmoid=False, renorm=False):
    l = np.asarray(logits, np.float64)
    T, E = l.shape
    s = scores(l, sigmoid)
    ids, w = np.zeros((T, k), np.int32), np.zeros((T, k))
    for t in range(T):
        c = s[t] + (0.0 if bias is None else np.asarray(bias, np.float64))
        c = np.where(l[t] == -np.inf, -np.inf, c)
        by = c if bias is not None else l[t]
        if top_groups < n_groups:
            best = -np.sort(-c.reshape(n_groups, -1), 1)[:, :group_top].sum(1)
            if bias is None and group_top == 1:
                best = l[t].reshape(n_groups, -1).max(1)
            out = np.ones(n_groups, bool)
            out[_order(best)[:top_groups]] = False
            open_ = np.flatnonzero(~np.repeat(out, E // n_groups))
        else:
            open_ = np.arange(E)
        ids[t] = open_[_order(by[open_])[:k]]
        p = s[t, ids[t]]
        if renorm:
            m = l[t, ids[t]].max()
            if sigmoid and m < -30 and np.isfinite(m):   # where sigmoids leave 64 bits' range their ratios do not
                p = np.exp(l[t, ids[t]] - m) / (1.0 + np.exp(l[t, ids[t]]))
            p = p / p.sum() if p.sum() > 0 else np.zeros(k)
        w[t] = p * scale
    return ids, w


def bwd(logits, ids, dw, scale=1.0, sigmoid=False, renorm=False):
    """-> gradient, and the size of what each entry is summed from"""
    l = np.asarray(logits, np.float64)
    T, E = l.shape
    s = scores(l, sigmoid)
    d, size = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        on = [(int(i), float(g) * scale) for i, g in zip(ids[t], np.asarray(dw, np.float64)[t]) if 0 <= i < E]
        if not on or all(g == 0 for _, g in on):
            continue
        i, g = np.array([x[0] for x in on]), np.array([x[1] for x in on])
        p = s[t, i]
        if renorm:
            m = l[t, i].max()
            q = np.exp(l[t, i] - m) / (1.0 + np.exp(l[t, i])) if sigmoid and m < -30 and np.isfinite(m) else p
            w = q / q.sum() if q.sum() > 0 else np.zeros(len(q))
            f = w * ((1.0 - p) if sigmoid else 1.0)
            np.add.at(d[t], i, f * (g - (g * w).sum()))
            np.add.at(size[t], i, f * 2 * np.abs(g - g[0]).max())
        elif sigmoid:
            np.add.at(d[t], i, g * p * (1.0 - p))
            np.add.at(size[t], i, np.abs(g) * p * (1.0 - p))
        else:
            d[t] -= s[t] * (g * p).sum()
            size[t] += s[t] * np.abs(g * p).sum()
            np.add.at(d[t], i, g * p)
            np.add.at(size[t], i, np.abs(g) * p)
    return d, size


def undecided(logits, bias, k, n_groups, top_groups, group_top, sigmoid):
    """Rows whose choice 64 bits do not settle: two neighbours in the order that decides, of different logits and biases, nearer than
    2^-46 of the largest score and 2^-51 of the largest c.  A score in 64 bits is off by under 2^-47 of itself (the exponential's unit, the
    argument's rounding, a sum of up to 1024 terms along 70 additions), c by 2^-53 more, a group's score by both twice."""
    if bias is None and not (top_groups < n_groups and group_top == 2):
        return np.zeros(len(logits), bool)
    l, s = np.asarray(logits, np.float64), scores(logits, sigmoid)
    b = np.zeros(l.shape[1]) if bias is None else np.asarray(bias, np.float64)
    out = np.zeros(len(l), bool)
    for t in range(len(l)):
        c = np.where(l[t] == -np.inf, -np.inf, s[t] + b)
        thr = 2.0 ** -46 * s[t].max() + 2.0 ** -51 * np.abs(c[np.isfinite(c)]).max(initial=0.0)
        near = lambda x, y: x == y or abs(x - y) <= 2 * thr
        pair = lambda e: (l[t, e], b[e]) if l[t, e] > -np.inf else (-np.inf, 0.0)   # a logit of -infinity: c is that, whatever the bias
        kept = np.ones(n_groups, bool)
        if top_groups < n_groups:
            rows = c.reshape(n_groups, -1)
            best = -np.sort(-rows, 1)[:, :group_top].sum(1)
            what = [sorted(pair(g * rows.shape[1] + i) for i in _order(rows[g])[:group_top]) for g in range(n_groups)]
            what = [(-np.inf,) if best[g] == -np.inf else what[g] for g in range(n_groups)]
            o = _order(best)
            border = best[o[top_groups - 1]]
            same = [g for g in range(n_groups) if near(best[g], border)]
            out[t] |= any(g in o[top_groups:] and what[g] != what[o[top_groups - 1]] for g in same) or \
                any(g in o[:top_groups] and what[g] != what[o[top_groups]] and near(best[g], best[o[top_groups]]) for g in range(n_groups))
            kept[o[top_groups:]] = False
        if bias is not None:
            open_ = np.flatnonzero(np.repeat(kept, l.shape[1] // n_groups))
            o = open_[_order(c[open_])][:k + 1]
            out[t] |= any(near(c[i], c[j]) and pair(i) != pair(j) for i, j in zip(o[:-1], o[1:]))
    return out
