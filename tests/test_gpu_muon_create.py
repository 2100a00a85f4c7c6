"""A handle made on a stream whose freed memory, still written by what is enqueued there, becomes its workspace."""
import pytest
import torch

from .test_gpu_muon import _bits, _gradient

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,rows,cols", [(2, 64, 96), (2, 200, 264)])
def test_made_behind_pending_work(n, rows, cols):
    from paper_2605_23764_b200 import MoeMuon
    G = _gradient(n, rows, cols, 1)
    first = MoeMuon(n, rows, cols)
    want, size = first.orthogonalize(G), first.workspace.numel()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        held = torch.empty(size, dtype=torch.uint8, device="cuda")
        at = held.data_ptr()
        torch.cuda._sleep(50_000_000)
        held.fill_(255)
        del held
        muon = MoeMuon(n, rows, cols)
        assert muon.workspace.data_ptr() == at
        out = muon.orthogonalize(G)
        assert muon.status() == (0, 0)
    side.synchronize()
    assert torch.equal(_bits(out), _bits(want))


def test_a_layer_made_behind_pending_work():
    from paper_2605_23764_b200 import MoeLayer
    T, d, E, k, F = 64, 128, 16, 2, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    x, logits = torch.randn(T, d, device="cuda", generator=g).to(torch.bfloat16), torch.randn(T, E, device="cuda", generator=g)
    W1 = (torch.randn(E, 2 * F, d, device="cuda", generator=g) / d ** 0.5).to(torch.bfloat16)
    W2 = (torch.randn(E, d, F, device="cuda", generator=g) / F ** 0.5).to(torch.bfloat16)
    first = MoeLayer(T, d, E, k, 0, F)
    ids, w = first.route(logits)
    want, size = first.ffn_fwd(x, ids, w, W1, W2), first.workspace.numel()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        held = torch.empty(size, dtype=torch.uint8, device="cuda")
        at = held.data_ptr()
        torch.cuda._sleep(50_000_000)
        held.fill_(255)
        del held
        layer = MoeLayer(T, d, E, k, 0, F)
        assert layer.workspace.data_ptr() == at
        out = layer.ffn_fwd(x, ids, w, W1, W2)
        assert layer.status() == (0, 0)
    side.synchronize()
    assert torch.equal(_bits(out), _bits(want))
