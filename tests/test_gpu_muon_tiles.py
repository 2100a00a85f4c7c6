"""Orthogonalised momentum of matrices that go through tiles (beyond 128 x 384, or 384 x 128): rows that are no whole vectors."""
import pytest
import torch

from .test_gpu_muon import _bits, _gradient

pytestmark = pytest.mark.gpu


def _shifted(t):
    """A copy that starts an element beyond an aligned address."""
    return torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape).copy_(t)


# one tile high with its reduction in parts, several boxes a warp, more tiles than pairs of SMs; wide and tall
@pytest.mark.parametrize("n,rows,cols", [(1, 256, 2056), (3, 520, 1000), (3, 1000, 520), (60, 264, 392), (60, 392, 264)])
@pytest.mark.parametrize("steps", [2, 5])
def test_unaligned_tensors_give_the_same_bits(n, rows, cols, steps):
    """Outputs that are no whole vectors leave through the same slots of shared memory that the next box's loads use."""
    from paper_2605_23764_b200 import MoeMuon
    muon = MoeMuon(n, rows, cols, steps=steps)
    W, M, dW = _gradient(n, rows, cols, 4, scale=0.1), _gradient(n, rows, cols, 6, torch.float32), _gradient(n, rows, cols, 5)
    want = muon.step(W, M, dW, 0.02, weight_decay=0.1, W_out=torch.empty_like(W), M_out=torch.empty_like(M))
    for _ in range(5):
        got = muon.step(_shifted(W), M, dW, 0.02, weight_decay=0.1, W_out=_shifted(W), M_out=torch.empty_like(M))
        assert got[0].data_ptr() % 16 and torch.equal(_bits(got[0]), _bits(want[0])) and torch.equal(_bits(got[1]), _bits(want[1]))
        assert torch.equal(_bits(muon.orthogonalize(dW, out=_shifted(W))), _bits(muon.orthogonalize(dW)))
    assert muon.status() == (0, 0)
