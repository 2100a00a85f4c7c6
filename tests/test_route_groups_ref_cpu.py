"""The 64-bit statement of routing by groups: its gradient is that of its weights, and its choice is the definition's."""
import numpy as np
import pytest
import torch

from . import route_groups_ref as R


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_is_that_of_the_weights(sigmoid, renorm):
    rng = np.random.default_rng(3)
    l = rng.normal(size=(20, 24)) * 2
    dw = rng.normal(size=(20, 5))
    ids, w = R.fwd(l, 5, rng.normal(size=24) * 0.1, 4, 2, 2, 2.5, sigmoid, renorm)
    x = torch.tensor(l, requires_grad=True)
    s = torch.sigmoid(x) if sigmoid else torch.softmax(x, 1)
    p = torch.gather(s, 1, torch.as_tensor(ids, dtype=torch.int64))
    p = (p / p.sum(1, keepdim=True) if renorm else p) * 2.5
    assert np.allclose(p.detach().numpy(), w, rtol=1e-12)
    (p * torch.tensor(dw)).sum().backward()
    assert np.allclose(R.bwd(l, ids, dw, 2.5, sigmoid, renorm)[0], x.grad.numpy(), atol=1e-14)
    # and against differences, where the choice stays
    h, e = 1e-6, 7
    up, down = l.copy(), l.copy()
    up[:, e] += h
    down[:, e] -= h
    pick = lambda v: sum(((lambda q: (q / q.sum() if renorm else q) * 2.5)(R.scores(v, sigmoid)[t, ids[t]]) * dw[t]).sum() for t in range(20))
    assert abs((pick(up) - pick(down)) / (2 * h) - R.bwd(l, ids, dw, 2.5, sigmoid, renorm)[0][:, e].sum()) < 1e-7


def test_groups_and_ties():
    l = np.zeros((1, 12))
    assert R.fwd(l, 4, None, 3, 2, 2)[0].tolist() == [[0, 1, 2, 3]]
    b = np.zeros(12)
    b[9] = 0.5
    assert R.fwd(l, 3, b, 3, 1, 2)[0].tolist() == [[9, 8, 10]]
    l[0, 8:] = -np.inf   # a group without a finite logit is never taken while others are left
    assert R.fwd(l, 8, b, 3, 2, 1)[0].max() < 8
