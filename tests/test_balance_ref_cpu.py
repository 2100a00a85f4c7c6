"""The 64-bit balance losses that the kernels are compared with, against differences and against the score gradient's oracle."""
import numpy as np
import pytest

import oracle

from . import balance_ref as R


def _objective(logits, ids, off, mask, dl, dw, sigmoid, renorm):
    losses, _, _, _ = R.fwd(logits, ids, off, mask, sigmoid)
    v = R.rows(logits, sigmoid)[2 if sigmoid else 1]
    w = np.take_along_axis(v, ids.astype(np.int64), 1)
    if renorm:
        w = w / w.sum(1, keepdims=True)
    return dl[0] * losses[0] + dl[1] * losses[1] + (w * dw).sum()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_against_differences(sigmoid, renorm):
    rng = np.random.default_rng(3)
    T, E, k = 11, 6, 2
    off, mask = [1, 4, 4, 10], np.array([1, 1, 0, 1, 1, 1, 1, 0, 1, 1, 1])
    logits = rng.normal(size=(T, E)) * 1.5
    ids = np.argsort(-logits, 1)[:, :k].astype(np.int32)
    dl, dw = np.array([0.7, -0.3]), rng.normal(size=(T, k))
    _, counts, _, tokens = R.fwd(logits, ids, off, mask, sigmoid)
    assert list(tokens) == [2, 0, 5, 7] and counts.sum() == 14
    grad, _ = R.bwd(logits, ids, counts, tokens, dl, dw, off, mask, sigmoid, renorm)
    h = 1e-5   # third derivatives of order one: the difference is off by h^2 and by 2^-52 / h
    for t in range(T):
        for e in range(E):
            up, down = logits.copy(), logits.copy()
            up[t, e] += h
            down[t, e] -= h
            num = (_objective(up, ids, off, mask, dl, dw, sigmoid, renorm) - _objective(down, ids, off, mask, dl, dw, sigmoid, renorm)) / (2 * h)
            assert abs(num - grad[t, e]) <= 1e-8, (t, e, num, grad[t, e])


@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_without_losses_it_is_the_score_gradient(gate, renorm):
    rng = np.random.default_rng(4)
    logits = rng.normal(size=(20, 9)).astype(np.float32)
    ids, _ = oracle.route(logits, 3, renorm, gate=gate)
    dw = rng.normal(size=(20, 3)).astype(np.float32)
    _, counts, _, tokens = R.fwd(logits, ids, sigmoid=gate == "sigmoid")
    d, _ = R.bwd(logits, ids, counts, tokens, [0.0, 0.0], dw, sigmoid=gate == "sigmoid", renorm=renorm)
    np.testing.assert_allclose(d, oracle.router_bwd(logits, ids, dw, renorm, gate=gate), atol=1e-12)


def test_even_routing_has_a_loss_of_one():
    E, k = 8, 2
    logits = np.zeros((E, E))
    ids = np.stack([np.arange(E), (np.arange(E) + 3) % E], 1)
    losses, counts, prob, tokens = R.fwd(logits, ids)
    assert np.isclose(losses[0], 1.0) and np.isclose(losses[1], np.log(E) ** 2)
    assert (counts == k).all() and np.allclose(prob, 1 / E) and list(tokens) == [E, E]
