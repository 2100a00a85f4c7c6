"""Biases that keep experts out of the choice, or in it, beside ordinary ones: the choice is the statement's, and the other experts' comparisons
cost what they cost without them.

Rows that 64 bits do not settle are left out: neighbours in the order that decides, of different logits or biases, that are nearer than what two c, or
two groups' scores, are off in 64 bits.  A score is off by under 2^-47 of itself (route_groups_ref.undecided), c by 2^-53 of itself more, a
group's score by its two c's and 2^-53 of itself: two values x, y by 2^-46 of the largest score and 2^-52 of the larger of |x|, |y|, groups by twice
the first and, for their larger c, 2^-51 of its magnitude.  (By the largest |c| of the row, as undecided() has it, one bias of -1e30 leaves every row open.)"""
import numpy as np
import pytest
import torch

from . import route_groups_ref as R
from .test_gpu_route_groups import _dev, _layer

pytestmark = pytest.mark.gpu
INF = float("inf")


def _bias(rng, E, sigmoid, values):
    b = (rng.integers(-100, 101, E) * 1e-3 * (1.0 if sigmoid else 0.05)).astype(np.float32)
    for i, e in enumerate(rng.permutation(E)[:max(1, E // 6)]):
        b[e] = values[i % len(values)]
    return b


def _open(l, b, k, n_groups, top_groups, group_top, sigmoid):
    """Whether 64 bits leave a row's choice open"""
    s = R.scores(l[None].astype(np.float64), sigmoid)[0]
    c = np.where(l == -np.inf, -np.inf, s + b.astype(np.float64))
    big = np.where(np.isfinite(c), np.abs(c), 0.0)
    kept = np.ones(n_groups, bool)
    if top_groups < n_groups:
        rows, size = c.reshape(n_groups, -1), big.reshape(n_groups, -1)
        top = np.argsort(-rows, 1, kind="stable")[:, :group_top]
        best = np.take_along_axis(rows, top, 1).sum(1)
        off = 2.0 ** -46 * s.max() + 2.0 ** -51 * np.take_along_axis(size, top, 1).max(1)
        o = np.argsort(-best, kind="stable")
        kept[o[top_groups:]] = False
        stays, goes = o[:top_groups], o[top_groups:]
        if (best[stays] - off[stays]).min() <= (best[goes] + off[goes]).max() and np.isfinite((best[goes] + off[goes]).max()):
            return True
    on = np.flatnonzero(np.repeat(kept, len(l) // n_groups))
    o = on[np.argsort(-c[on], kind="stable")][:k + 1]
    x, y = o[:-1], o[1:]
    with np.errstate(invalid="ignore"):   # -infinity beside -infinity: the lower one, no doubt
        near = c[x] - c[y] <= 2.0 ** -46 * s.max() + 2.0 ** -52 * np.maximum(big[x], big[y])
    return bool((near & ((l[x] != l[y]) | (b[x] != b[y]))).any())


def _check(logits, k, bias, groups, sigmoid, renorm):
    layer = _layer(logits.shape[0], logits.shape[1], k, sigmoid, renorm)
    ids, w, counts = layer.route_grouped(_dev(logits), _dev(bias), *groups, with_counts=True)
    ids = ids.cpu().numpy()
    want, _ = R.fwd(logits, k, bias, *groups, sigmoid=sigmoid, renorm=renorm)
    left_out = np.array([_open(l, bias, k, *groups[:3], sigmoid) for l in logits])
    assert left_out.sum() <= 1 + len(logits) // 8
    assert np.array_equal(ids[~left_out], want[~left_out]), np.flatnonzero((ids != want).any(1) & ~left_out)[:5]
    assert torch.isfinite(w).all() and layer.status() == (0, 0)
    assert np.array_equal(counts.cpu().numpy(), np.bincount(ids.reshape(-1), minlength=logits.shape[1]))


@pytest.mark.parametrize("values", [(-INF,), (-1e9,), (-1e30, -INF, -3e38), (1e4, -1e4), (1e9, -1e9, -INF)])
@pytest.mark.parametrize("E,k,groups", [(256, 8, (8, 4, 2, 2.5)), (160, 6, (10, 4, 2, 1.0)), (96, 5, (4, 2, 1, 1.0)), (512, 10, (1, 1, 1, 1.0)), (64, 6, (32, 7, 2, 1.0))])
@pytest.mark.parametrize("sigmoid", [True, False])
def test_choice(values, E, k, groups, sigmoid):
    rng = np.random.default_rng(E)
    logits = (rng.normal(size=(300, E)) * 1.7).astype(np.float32)
    logits[200:250][rng.random((50, E)) < 0.6] = -np.inf
    logits[::7] = np.round(logits[::7])
    _check(logits, k, _bias(rng, E, sigmoid, values), groups, sigmoid, True)


def test_all_but_k_experts_kept_out():
    rng = np.random.default_rng(4)
    b = np.full(64, -INF, np.float32)
    b[[3, 17, 18, 40, 41, 62]] = 0.125
    _check((rng.normal(size=(200, 64))).astype(np.float32), 6, b, (1, 1, 1, 1.0), True, True)
    b[[0, 1]] = -1e9
    _check((rng.normal(size=(200, 64))).astype(np.float32), 6, b, (4, 3, 1, 1.0), True, True)


@pytest.mark.parametrize("value", [-INF, -1e9])
def test_the_others_are_not_settled_in_64_bits(value):
    """Time beside the same call without: 64 bits for every token are six times as long."""
    T, E, k = 32768, 256, 8
    layer = _layer(T, E, k, True, True)
    rng = np.random.default_rng(0)
    logits = _dev(rng.normal(size=(T, E)) * 1.7, torch.float32)
    plain = _dev(rng.integers(-100, 101, E) * 1e-3, torch.float32)
    out = plain.clone()
    out[[17, 99]] = value

    def time(bias):
        took = []
        for _ in range(9):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(4):
                layer.route_grouped(logits, bias, 8, 4, 2)
            b.record()
            torch.cuda.synchronize()
            took.append(a.elapsed_time(b))
        return sorted(took)[4]
    time(plain)
    assert time(out) < 2.5 * time(plain)
