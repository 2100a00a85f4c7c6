"""Padding of a batch in a training step: the scores' gradient is given, and is zero for padding, whose logits hold anything."""
import numpy as np
import pytest

from .test_gpu_balance import _case, _check, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sigmoid,renorm", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("E,k", [(8, 3), (40, 6), (41, 4), (256, 8), (512, 2)])
def test_padding_without_a_score_gradient_holds_anything(E, k, sigmoid, renorm):
    T = 90
    logits, ids, dw = _case(T, E, k, 15 + E)
    mask = np.ones(T, np.uint8)
    mask[5:17] = 0
    off = np.array([3, 40, 80], np.int32)
    idle = (mask == 0) | (np.arange(T) < 3) | (np.arange(T) >= 80)
    dw[idle] = 0
    opt = dict(off=off, mask=mask, renorm=renorm, sigmoid=sigmoid)
    clean = [g.copy() for g in _run(logits, ids, dw, **opt)]
    _check(clean, logits, ids, dw, **opt)
    assert not clean[4][idle].any()
    for v in (np.nan, np.inf, -np.inf):
        logits[idle] = v
        logits[7, ::2] = 1.0
        for want, got in zip(clean, _run(logits, ids, dw, **opt)):
            assert np.array_equal(want, got)
        ids[idle] = E + 5   # nor does it matter what padding names
        dw[idle, 0] = 1.0   # (what arrives for an id that is none is no gradient)
        for want, got in zip(clean, _run(logits, ids, dw, **opt)):
            assert np.array_equal(want, got)
        ids[idle], dw[idle] = 1, 0


@pytest.mark.parametrize("sigmoid", [False, True])
def test_padding_with_a_score_gradient_still_gets_it(sigmoid):
    """One slot of the last ones alone has a gradient: a token that takes no part keeps it."""
    T, E, k = 64, 24, 6
    logits, ids, dw = _case(T, E, k, 2)
    mask = (np.arange(T) % 3 > 0).astype(np.uint8)
    dw[mask == 0, :k - 1] = 0
    for renorm in (False, True):
        got = _run(logits, ids, dw, mask=mask, renorm=renorm, sigmoid=sigmoid)
        _check(got, logits, ids, dw, mask=mask, renorm=renorm, sigmoid=sigmoid)
        assert (np.abs(got[4][mask == 0]).max(1) > 0).all()
