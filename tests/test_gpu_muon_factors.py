"""Factors of an update that are finite numbers whose products are not: refused, and nothing is written."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(16, 24), (130, 200)])
@pytest.mark.parametrize("bad", [dict(lr=1e30, scale=1e30), dict(lr=1e30, weight_decay=1e30), dict(lr=-1e20, scale=1e20)])
def test_products_beyond_fp32_are_refused(rows, cols, bad):
    from paper_2605_23764_b200 import MoeError, MoeMuon
    muon = MoeMuon(1, rows, cols)
    W, M, dW = torch.ones(1, rows, cols, dtype=torch.bfloat16, device="cuda"), torch.ones(1, rows, cols, device="cuda"), \
        torch.ones(1, rows, cols, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(MoeError):
        muon.step(W, M, dW, **bad)
    torch.cuda.synchronize()
    assert bool((W == 1).all()) and bool((M == 1).all())
    muon.step(W, M, dW, lr=1e10, scale=1e-12)
    assert torch.isfinite(W).all() and muon.status() == (0, 0)
