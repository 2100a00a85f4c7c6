"""Routing by groups where fp32 cannot order what decides: scores far below 1, whose relative error grows with the logits.  Rows that 64 bits do
not settle either are left out (undecided()); everything else has to be the statement's."""
import numpy as np
import pytest
import torch

from . import route_groups_ref as R
from .test_gpu_route_groups import _dev, _layer

pytestmark = pytest.mark.gpu


def _rows(rng, T, E, centre, steps):
    """fp32 neighbours of `centre`, up to `steps` away"""
    ulp = float(np.spacing(np.float32(abs(centre))))
    return (np.float64(centre) + rng.integers(-steps, steps + 1, (T, E)) * ulp).astype(np.float32), ulp


def _ids(logits, bias, k, groups):
    layer = _layer(logits.shape[0], logits.shape[1], k, True, True)
    ids, _ = layer.route_grouped(_dev(logits), _dev(bias), *groups)
    return ids.cpu().numpy()


def _check_ids(logits, bias, k, groups):
    ids = _ids(logits, bias, k, groups)
    want, _ = R.fwd(logits, k, bias, *groups, sigmoid=True, renorm=True)
    wrong = (ids != want).any(1)
    wrong[wrong] = ~R.undecided(logits[wrong], None if bias is None else bias, k, *groups, True)   # few rows: this is slow
    assert not wrong.any(), (int(wrong.sum()), np.flatnonzero(wrong)[:5])


@pytest.mark.parametrize("centre", [-2.0, -8.0, -12.0, -20.0, -25.0, -30.0, -40.0, -60.0, -70.0, -85.0])
@pytest.mark.parametrize("steps", [6, 40])
def test_groups_by_the_sum_of_two_small_scores(centre, steps):
    rng = np.random.default_rng(int(-centre) + steps)
    logits, _ = _rows(rng, 8000, 256, centre, steps)
    _check_ids(logits, None, 8, (8, 4, 2))


@pytest.mark.parametrize("centre", [-2.0, -8.0, -12.0, -20.0, -30.0, -40.0, -60.0, -80.0])
@pytest.mark.parametrize("groups", [(1, 1, 1), (4, 2, 1)])
def test_biases_that_undo_differences_of_small_scores(centre, groups):
    """Biases as small as the scores, whole numbers of a logit's step of them: sums of the two meet but for terms of second order."""
    rng = np.random.default_rng(int(-centre))
    logits, ulp = _rows(rng, 8000, 64, centre, 3)
    bias = (rng.integers(-3, 4, 64) * (np.exp(centre) * ulp)).astype(np.float32)
    _check_ids(logits, bias, 6, groups)
