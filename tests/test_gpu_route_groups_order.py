"""Without a bias experts go by their logits, and groups by their best expert (group_top = 1) do too: also where scores are equal in 64 bits, sigmoids
of 40 and 50, softmax scores 800 behind the largest.  Groups by the sum of two scores, and all with a bias, go by the scores."""
import numpy as np
import pytest

from . import route_groups_ref as R
from .test_gpu_route_groups import _dev, _layer

pytestmark = pytest.mark.gpu


def _ids(logits, k, bias, groups, sigmoid):
    ids, _ = _layer(*logits.shape, k, sigmoid, True).route_grouped(_dev(logits), _dev(bias), *groups)
    return ids.cpu().numpy()


@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("E,k,G,top", [(256, 8, 8, 4), (40, 4, 10, 3), (64, 2, 32, 5)])
def test_equal_scores(sigmoid, E, k, G, top):
    rng = np.random.default_rng(E)
    logits = (40 + rng.uniform(0, 20, (100, E)) if sigmoid else rng.uniform(-1000, -800, (100, E))).astype(np.float32)
    if not sigmoid:
        logits[:, 0] = 0.0
    gs = E // G
    best = logits.reshape(100, G, gs).max(2)
    order = np.argsort(-best, 1, kind="stable")
    by_logit = np.full(logits.shape, -np.inf)
    by_index = np.full(logits.shape, -np.inf)
    for t in range(100):
        for g in range(top):
            s = slice(order[t, g] * gs, order[t, g] * gs + gs)
            by_logit[t, s] = logits[t, s]
            s = slice(g * gs, g * gs + gs)      # equal sums: the lowest groups (with a softmax the first one is the largest)
            by_index[t, s] = logits[t, s]
    want = np.argsort(-by_logit, 1, kind="stable")[:, :k]
    assert np.array_equal(_ids(logits, k, None, (G, top, 1), sigmoid), want)
    want = np.argsort(-by_index, 1, kind="stable")[:, :k]
    assert np.array_equal(_ids(logits, k, None, (G, top, 2), sigmoid), want)
    assert np.array_equal(R.fwd(logits, k, None, G, top, 2, sigmoid=sigmoid)[0], want)
    zeros = np.zeros(E, np.float32)             # a bias: scores decide, equal ones by index
    assert np.array_equal(_ids(logits, k, zeros, (G, top, 1), sigmoid), np.tile(np.arange(k), (100, 1)))
