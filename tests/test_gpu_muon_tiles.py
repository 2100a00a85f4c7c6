"""Orthogonalised momentum of matrices that go through tiles (beyond 128 x 384, or 384 x 128): rows that are no whole vectors, other polynomials,
numbers that are none, updates in place, few steps, captures, a layer's training step.  Tolerances as in test_gpu_muon.py."""
import numpy as np
import pytest
import torch

from .test_gpu_muon import BF16, COEF, NORM, _bits, _exact, _gradient, _near

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


@pytest.mark.parametrize("coef,steps", [(COEF, 1), (COEF, 2), (COEF, 3), (COEF, 4), (COEF, 7), ((1.5, -0.5, 0.0), 12), ((1.875, -1.25, 0.375), 8),
                                        ([(4.0, -7.0, 3.5), (3.5, -5.0, 2.2), (1.875, -1.25, 0.375)], 3)])
@pytest.mark.parametrize("n,rows,cols", [(3, 256, 400), (2, 400, 264), (2, 300, 300), (1, 192, 1100), (1, 131, 523)])
def test_other_polynomials(coef, steps, n, rows, cols):
    from paper_2605_23764_b200 import MoeMuon
    G = _gradient(n, rows, cols, steps)
    _near(MoeMuon(n, rows, cols, coefficients=coef, steps=steps).orthogonalize(G), _exact(G, coef, steps))


@pytest.mark.parametrize("rows,cols", [(200, 456), (456, 200), (133, 401), (256, 2056)])
def test_scale_zeros_and_faults_stay_in_their_matrix(rows, cols):
    from paper_2605_23764_b200 import MoeMuon
    G = _gradient(6, rows, cols, 1, torch.float32, 1.0)
    muon = MoeMuon(6, rows, cols, eps=0.0)
    plain = muon.orthogonalize(G)
    mixed = G * torch.tensor([2.0 ** -90, 2.0 ** 90, 1.0, 0.0, 1.0, 1.0], device="cuda")[:, None, None]
    mixed[4, 3, 5] = float("nan")
    mixed[5, 0, 0] = float("inf")
    out = muon.orthogonalize(mixed)
    assert torch.equal(_bits(out[:3]), _bits(plain[:3]))       # powers of two change no bit
    assert not out[3].any()
    assert torch.isnan(out[4]).all() and torch.isnan(out[5]).all() and muon.status() == (0, 0)
    assert torch.equal(_bits(muon.orthogonalize(G)), _bits(plain))   # nothing of it stays in the workspace
    assert not MoeMuon(6, rows, cols).orthogonalize(torch.zeros_like(G)).any()


# up to three steps: the last step reads W from memory, later ones load it beside X
@pytest.mark.parametrize("steps", [1, 2, 3, 5])
@pytest.mark.parametrize("n,rows,cols", [(3, 256, 400), (2, 400, 256), (1, 256, 2056), (40, 264, 392), (2, 131, 401)])
@pytest.mark.parametrize("nesterov", [True, False])
def test_step(n, rows, cols, steps, nesterov):
    from paper_2605_23764_b200 import MoeMuon
    g = torch.Generator(device="cuda").manual_seed(rows)
    W = (torch.randn(n, rows, cols, device="cuda", generator=g) * 0.1).to(torch.bfloat16)
    dW, M = _gradient(n, rows, cols, 5), _gradient(n, rows, cols, 6, torch.float32, 1e-3)
    mu, lr, wd, scale = np.float32(0.9), np.float32(0.02), np.float32(0.1), np.float32(1.5)
    muon = MoeMuon(n, rows, cols, momentum=0.9, nesterov=nesterov, steps=steps)
    W1, M1 = muon.step(W, M, dW, lr=0.02, weight_decay=0.1, scale=1.5, W_out=torch.empty_like(W), M_out=torch.empty_like(M))
    m = float(mu) * M.double() + dW.double()
    assert bool(((M1.double() - m).abs() <= 2.0 ** -24 * m.abs() + 1e-44).all())
    x = _exact(dW.double() + float(mu) * m if nesterov else m, steps=steps)
    rate = float(lr) * float(scale)
    want = (1 - float(lr) * float(wd)) * W.double() - rate * x
    rms = x.flatten(1).norm(dim=1) / (rows * cols) ** 0.5
    assert bool(((W1.double() - want).abs() <= rate * 10 * NORM * rms[:, None, None] + (BF16 + 3 * 2.0 ** -24) * (want.abs() + rate * x.abs())).all())
    W2, M2 = W.clone(), M.clone()
    got = muon.step(W2, M2, dW, lr=0.02, weight_decay=0.1, scale=1.5)   # in place
    assert got[0] is W2 and got[1] is M2 and torch.equal(_bits(W2), _bits(W1)) and torch.equal(_bits(M2), _bits(M1))
    assert muon.status() == (0, 0)


def test_step_of_more_matrices_than_the_workspace_holds():
    """Every matrix gets what it gets alone, weights and momentum, in place."""
    from paper_2605_23764_b200 import MoeMuon
    n, rows, cols = 70, 1024, 1536
    W, M, dW = _gradient(n, rows, cols, 1, scale=0.1), _gradient(n, rows, cols, 2, torch.float32), _gradient(n, rows, cols, 3)
    muon, one = MoeMuon(n, rows, cols), MoeMuon(1, rows, cols)
    old_W, old_M = W.clone(), M.clone()
    muon.step(W, M, dW, 0.01)
    assert muon.launches() > 3
    for i in (0, 33, 34, 46, 47, 69):
        a, b = one.step(old_W[i:i + 1], old_M[i:i + 1], dW[i:i + 1], 0.01, W_out=torch.empty_like(W[:1]), M_out=torch.empty_like(M[:1]))
        assert torch.equal(_bits(W[i]), _bits(a[0])) and torch.equal(_bits(M[i]), _bits(b[0])), i


@pytest.mark.parametrize("n,rows,cols", [(3, 200, 520), (1, 256, 2056), (2, 521, 203)])
def test_captured_and_replayed(n, rows, cols):
    from paper_2605_23764_b200 import MoeMuon
    W, M, dW = _gradient(n, rows, cols, 1, scale=0.1), _gradient(n, rows, cols, 2, torch.float32), _gradient(n, rows, cols, 3)
    muon = MoeMuon(n, rows, cols)
    We, Me = W.clone(), M.clone()
    for _ in range(3):
        muon.step(We, Me, dW, 0.01)
    graph = torch.cuda.CUDAGraph()
    Wg, Mg = W.clone(), M.clone()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        muon.step(Wg, Mg, dW, 0.01)
    assert torch.equal(Wg, W)
    for _ in range(3):
        graph.replay()
        muon.orthogonalize(dW)   # an eager call between two replays, on the same stream
    torch.cuda.synchronize()
    assert torch.equal(_bits(Wg), _bits(We)) and torch.equal(_bits(Mg), _bits(Me)) and muon.status() == (0, 0)


def test_a_layers_training_step():
    """As test_gpu_muon.py's, of matrices that go through tiles: both weight tensors, gate and up by themselves, an expert without tokens."""
    from paper_2605_23764_b200 import MoeLayer, MoeMuon
    T, d, E, k, S, F = 96, 512, 12, 2, 1, 160
    g = torch.Generator().manual_seed(4)
    layer = MoeLayer(T, d, E, k, S, F, renorm=True, sigmoid_gate=True, save_for_bwd=True)
    x = torch.randn(T, d, generator=g).to(torch.bfloat16).cuda()
    W1 = (torch.randn(E + S, 2 * F, d, generator=g) / d ** 0.5).to(torch.bfloat16).cuda()
    W2 = (torch.randn(E + S, d, F, generator=g) / F ** 0.5).to(torch.bfloat16).cuda()
    logits = torch.randn(T, E, generator=g).cuda()
    bias = torch.zeros(E, device="cuda")
    bias[5] = -float("inf")
    up, down = MoeMuon.for_gate_up(layer), MoeMuon.for_down(layer)
    M1, M2 = torch.zeros(W1.shape, device="cuda"), torch.zeros(W2.shape, device="cuda")
    for _ in range(2):
        ids, w = layer.route_grouped(logits, bias, 4, 2, 2, 2.5)
        out = layer.ffn_fwd(x, ids, w, W1, W2)
        dx, dW1, dW2, dw = layer.ffn_bwd(out, x, ids, w, W1, W2)
        old1, old2, m1, m2 = W1.clone(), W2.clone(), M1.double(), M2.double()
        up.step(W1, M1, dW1, lr=0.01, scale=0.5)
        down.step(W2, M2, dW2, lr=0.01, scale=0.5)
        assert layer.status() == (0, 0) and up.status() == (0, 0) and down.status() == (0, 0)
        assert not bool((ids == 5).any()) and torch.equal(W1[5], old1[5]) and torch.equal(W2[5], old2[5]) and not dW1[5].any()
        for W, old, m, dW, shape in ((W1, old1, m1, dW1, (2 * (E + S), F, d)), (W2, old2, m2, dW2, (E + S, d, F))):
            m = 0.95 * m + dW.double()
            x_ = _exact((dW.double() + 0.95 * m).view(shape)).view(W.shape)
            want = old.double() - 0.005 * x_
            assert bool(((W.double() - want).abs() <= 0.005 * 10 * NORM * x_.abs().amax() + BF16 * (want.abs() + 0.005 * x_.abs())).all())
        assert not torch.equal(W2[0], old2[0])
