"""Batches of which no slot names an expert: padding that a caller marks by ids out of range."""
import numpy as np
import pytest
import torch

from . import w4_ref as R
from .test_gpu_w4 import BF, _cuda, _problem, _weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S", [0, 1])
@pytest.mark.parametrize("T", [1, 3, 150, 400])
def test_no_slot_names_an_expert(T, S):
    """Zeros, or the shared experts alone; the next call is a whole one."""
    from paper_2605_23764_b200 import MoeLayer
    d, E, k, F, group = 136, 5, 2, 72, 64
    x, ids, w, up, down = _problem(T, d, E, k, S, F, group, True, T + S)
    W1, W2 = _weights(up, down, group)
    layer = MoeLayer(T, d, E, k, S, F, w4=True)
    none = np.full_like(ids, -1)
    none[::2] = E
    for named in (none, ids, none):
        out = layer.ffn_fwd_w4(_cuda(x, BF), _cuda(named), _cuda(w), W1, W2)
        torch.cuda.synchronize()
        assert layer.status()[0] == (1 if named is none else 0)   # MOE_ERR_BAD_EXPERT_ID
        want, bound = R.layer(x, named, w, R.values(*up, group), R.values(*down, group), E, rounded_weights=True)
        got = out.float().cpu().numpy()
        assert (np.abs(got - want) <= bound).all()
        if named is none and not S:
            assert not got.any()
    layer.close()
