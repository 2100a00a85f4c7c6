"""What the layer's accuracy tests can see: the limit in the norm lies between two roundings and rounded weights."""
import numpy as np
import pytest

from . import w4_ref as R


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("T", [2, 64])
def test_the_limit_lies_between_two_roundings_and_rounded_weights(T, asym):
    d, F, E, k, group = 1024, 512, 4, 2, 128
    rng = np.random.default_rng(T)
    x, w = R.bf16(rng.normal(size=(T, d))), rng.random((T, k)).astype(np.float32)
    ids = np.argsort(rng.random((T, E)), 1)[:, :k]
    W1, W2 = (R.values(*R.random_codes(rng, E, *shape, group, asym), group) for shape in ((2 * F, d), (d, F)))

    def layer(W1, W2, act=lambda a: a, out=lambda y: y):
        y = np.zeros((T, d))
        for e in range(E):
            t, j = np.nonzero(ids == e)
            h = x[t] @ W1[e].T
            g, u = h[:, :F], h[:, F:]
            np.add.at(y, t, act(w[t, j].astype(np.float64)[:, None] * g / (1 + np.exp(-g)) * u) @ W2[e].T)
        return out(y)

    want = layer(W1, W2)
    error = lambda y: np.linalg.norm(y - want) / np.linalg.norm(want)
    bf16 = lambda a: R.bf16(a).astype(np.float64)
    # 2.8e-3: test_gpu_w4_accuracy.py derives it
    assert error(layer(W1, W2, bf16, bf16)) < 2.8e-3
    assert error(layer(bf16(W1), bf16(W2), bf16, bf16)) > 2.8e-3
