"""The layer over 4-bit weights rounds activations and results to bf16, and no weight: to tolerances that rounded weights exceed.

Norm.  Rounding a number of significand m (1 <= m < 2) to bf16 is off by 2^-8 / (sqrt(3) m) of it in the mean square.  Over the values of a
tensor 1 / m^2 counts with the value's square, so that the mean square is 2^-16 / (3 M), M the mean of m^2: 2.2 where m is spread
logarithmically, 2.3 evenly.  M >= 1.3 holds for all but values that crowd above powers of two; two roundings, of the activation and of the
result, then are sqrt(2 / 3.9) 2^-8 = 2.8e-3 in the norm.  Weights rounded to bf16 are a third and a fourth one.

Elements.  As w4_ref.layer without rounded weights, and with what few tokens cost: there a group's sum is taken over 16 + q, and 16 + z times
the sum of x off it.  Each of the eight steps of either chain is off by two units of 2^-23 of a sum of at most 31 |x|: 2 x 8 x 2 x 31 = 992."""
import numpy as np
import pytest

from . import w4_ref as R
from .test_gpu_w4 import _run

pytestmark = pytest.mark.gpu
V = 2.0 ** -23


def _codes(rng, n, rows, cols, group, asym, most, share):
    """Codes up to `most` from the zero point, `share` of them not at it."""
    groups = -(-cols // group)
    z = rng.integers(most, 16 - most, size=(n, rows, groups)) if asym else np.full((n, rows, groups), 8)
    q = z[..., np.arange(cols) // group] + np.where(rng.random((n, rows, cols)) < share, rng.integers(-most, most + 1, size=(n, rows, cols)), 0)
    q = q.astype(np.uint8)
    s = R.bf16((rng.random((n, rows, groups)) + 0.5) * cols ** -0.5 / 4.6)
    return q[..., 0::2] | (q[..., 1::2] << 4), s, z.astype(np.uint8) if asym else None


def _layer(x, ids, w, up, down, group, E):
    """w4_ref.layer, its bound widened by the sums over 16 + q"""
    W1, W2 = R.values(*up, group), R.values(*down, group)
    want, bound = R.layer(x, ids, w, W1, W2, E)
    of = lambda cols: np.arange(cols) // group
    s1, s2 = up[1].astype(np.float64)[..., of(x.shape[1])], down[1].astype(np.float64)[..., of(W2.shape[2])]
    F = W2.shape[2]
    for e in range(W1.shape[0]):
        t, j = np.nonzero(ids == e)
        if not len(t):
            continue
        we = np.abs(w[t, j].astype(np.float64))[:, None]
        h, dh = x[t] @ W1[e].T, 992 * V * (np.abs(x[t]) @ s1[e].T)
        g, u = h[:, :F], h[:, F:]
        silu = g / (1 + np.exp(-g))
        da = we * (1.1 * dh[:, :F] * (np.abs(u) + dh[:, F:]) + np.abs(silu) * dh[:, F:])
        np.add.at(bound, t, 1.02 * (da @ np.abs(W2[e]).T + 992 * V * ((we * np.abs(silu * u) + da) @ s2[e].T)))
    return want, bound


def _tokens(rng, T, E, k):
    return np.argsort(rng.random((T, E)), 1)[:, :k].astype(np.int32), rng.random((T, k)).astype(np.float32)


@pytest.mark.parametrize("most,share", [(7, 1.0), (1, 1.0), (1, 1 / 16), (7, 1 / 64)])
@pytest.mark.parametrize("offset", [0.0, 1.0, 10.0])
@pytest.mark.parametrize("asym,group", [(True, 128), (False, 128), (True, 32)])
@pytest.mark.parametrize("T", [2, 64])   # one kernel, the other
def test_no_weight_is_rounded(T, asym, group, offset, most, share):
    """x with and without what all its elements have in common; codes spread over the range, next to the zero point, mostly at it."""
    d, F, E, k = 2048, 512, 4, 2
    rng = np.random.default_rng(17)
    x = R.bf16(offset + rng.normal(size=(T, d)))
    up, down = _codes(rng, E, 2 * F, d, group, asym, most, share), _codes(rng, E, d, F, group, asym, most, share)
    ids, w = _tokens(rng, T, E, k)
    got = _run(T, d, E, k, 0, F, x, ids, w, up, down, group)
    want, bound = _layer(x, ids, w, up, down, group, E)
    assert (np.abs(got - want) <= bound).all()
    off = np.linalg.norm(got - want) / np.linalg.norm(want)
    assert off <= 2.8e-3, off


@pytest.mark.parametrize("asym,group", [(False, 128), (True, 128), (True, 64)])
@pytest.mark.parametrize("T", [1, 48])
def test_large_x_with_small_scales(T, asym, group):
    """x up to 2^115, all of one sign: the largest sums that are taken on the way."""
    d, F, E, k = 1024, 128, 4, 2
    rng = np.random.default_rng(3)
    x = R.bf16((1 + rng.random((T, d))) * 2.0 ** 114)
    q, s, z = _codes(rng, E, 2 * F, d, group, asym, 7, 1.0)
    up = (q, R.bf16(s * np.float32(2.0 ** -115)), z)
    down = _codes(rng, E, d, F, group, asym, 7, 1.0)
    ids, w = _tokens(rng, T, E, k)
    got = _run(T, d, E, k, 0, F, x, ids, w, up, down, group)
    want, bound = _layer(x, ids, w, up, down, group, E)
    assert np.isfinite(got).all() and (np.abs(got - want) <= bound).all()
