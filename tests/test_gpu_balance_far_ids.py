"""Renormalised scores of experts that are far from the row's largest logit: ids may come from a selection of the caller's own (groups,
a bias), so that none of them need be near it."""
import numpy as np
import pytest

from .test_gpu_balance import _check, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("E,k", [(64, 2), (41, 3), (300, 8), (8, 1)])
@pytest.mark.parametrize("depth", [20.0, 60.0, 86.0])
def test_scores_of_experts_far_below_the_largest(E, k, depth):
    """At 86 below, a term of the softmax is a normal fp32 number, while divided by the sum of many experts it is none: the reciprocal of the
    scores' sum then is infinite."""
    T = 40
    rng = np.random.default_rng(E + k)
    logits = (rng.random((T, E)) * 0.5).astype(np.float32)
    ids = np.argsort(rng.random((T, E)), 1)[:, :k].astype(np.int32)
    np.put_along_axis(logits, ids.astype(np.int64), (0.5 - depth - rng.random((T, k)) * 0.5).astype(np.float32), 1)
    dw = rng.normal(size=(T, k)).astype(np.float32)
    for dl in ((0.0, 0.0), (0.02, 0.003)):
        got = _run(logits, ids, dw, renorm=True, dl=dl)
        assert np.isfinite(got[4]).all()
        _check(got, logits, ids, dw, renorm=True, dl=dl)
