"""Renormalised sigmoids far apart and far below 1: the small ones' shares of the sum are fp32 numbers although the scores are not."""
import numpy as np
import pytest

from .test_gpu_route_groups import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("top", [5.0, 0.0, -1.0, -30.0, -59.0, -61.0, -80.0, -200.0, -1000.0])
@pytest.mark.parametrize("E,k", [(16, 6), (256, 8)])
def test_shares_of_the_sum(top, E, k):
    rng = np.random.default_rng(E)
    logits = (top - rng.uniform(0, 60, (60, E))).astype(np.float32)
    logits[np.arange(60), rng.integers(0, E, 60)] = top
    logits[:30, k // 2:] = (top - rng.uniform(35, 60, (30, E - k // 2))).astype(np.float32)   # two or three experts, the others far behind
    _check(logits, k, None, (1, 1, 1, 2.5), True, True)
