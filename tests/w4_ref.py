"""4-bit weights and the layer over them, in numpy and 64 bits."""
import numpy as np
import torch


def bf16(v):
    return torch.from_numpy(np.ascontiguousarray(v, np.float32)).to(torch.bfloat16).float().numpy()


def random_codes(rng, n, rows, cols, group, asym):
    """natural codes [n][rows][cols / 2], scales [n][rows][groups] (fp32 values of bf16 numbers), zero points or None"""
    groups = -(-cols // group)
    q = rng.integers(0, 256, size=(n, rows, cols // 2), dtype=np.uint8)
    s = bf16((rng.random((n, rows, groups)) + 0.5) * cols ** -0.5 / 4.6)
    z = rng.integers(0, 16, size=(n, rows, groups), dtype=np.uint8) if asym else None
    return q, s, z


def values(q, s, z, group):
    """s (q - z) in 64 bits, exact"""
    cols = 2 * q.shape[2]
    v = np.empty(q.shape[:2] + (cols,))
    v[..., 0::2], v[..., 1::2] = q & 15, q >> 4
    of = np.arange(cols) // group
    return s.astype(np.float64)[..., of] * (v - (8.0 if z is None else z.astype(np.float64)[..., of]))


def quantized(W, group, asym):
    """The values that a bf16 matrix [n][rows][cols] becomes, by the definition, in fp32 with IEEE division"""
    f = np.float32
    out = np.empty(W.shape, np.float64)
    for a in range(0, W.shape[2], group):
        v = W[:, :, a:a + group].astype(f)
        if asym:
            lo, hi = np.minimum(v.min(2, keepdims=True), f(0)), np.maximum(v.max(2, keepdims=True), f(0))
            s = bf16((hi - lo) / f(15))
            step = np.where(s > 0, s, f(1))
            z = np.clip(np.rint(-lo / step), 0, 15)
            q = np.clip(np.rint(v / step) + z, 0, 15)
        else:
            s = bf16(np.abs(v).max(2, keepdims=True) / f(7))
            z = f(8)
            q = np.clip(np.rint(v / np.where(s > 0, s, f(1))) + f(8), 0, 15)
        out[:, :, a:a + group] = s.astype(np.float64) * (q - z).astype(np.float64)
    return out


def layer(x, ids, w, W1, W2, E, rounded_weights=False):
    """out, and a bound of the error of bf16 activations between fp32 products, element by element.

    U = 2^-8 is a bf16 rounding.  A product of K terms in fp32 is off by at most (K + 8) 2^-23 sum |x W|; SwiGLU by 2^-18 of its
    result (approximate exponential and quotient); the activation is rounded to bf16 once, the result once.  rounded_weights: the
    weights themselves are rounded to bf16 as well."""
    T, d = x.shape
    F = W2.shape[2]
    U, V = 2.0 ** -8, 2.0 ** -23
    wr = U if rounded_weights else 0.0
    out, bound = np.zeros((T, d)), np.zeros((T, d))
    for e in range(W1.shape[0]):
        if e < E:
            t, j = np.nonzero(ids == e)
            we = w[t, j].astype(np.float64)
        else:
            t, we = np.arange(T), np.ones(T)
        if not len(t):
            continue
        h, ha = x[t] @ W1[e].T, np.abs(x[t]) @ np.abs(W1[e]).T
        g, u = h[:, :F], h[:, F:]
        dg, du = ((d + 8) * V + wr) * ha[:, :F], ((d + 8) * V + wr) * ha[:, F:]
        silu = g / (1 + np.exp(-g))
        a = we[:, None] * silu * u
        da = np.abs(we)[:, None] * (1.1 * dg * (np.abs(u) + du) + np.abs(silu) * du) + 2.0 ** -18 * np.abs(a)
        da += U * (np.abs(a) + da)
        np.add.at(out, t, a @ W2[e].T)
        np.add.at(bound, t, da @ np.abs(W2[e]).T + ((F + 8) * V + wr) * ((np.abs(a) + da) @ np.abs(W2[e]).T))
    return out, (1 + U) * bound + U * np.abs(out) + 64 * V * np.abs(out) + 1e-30
