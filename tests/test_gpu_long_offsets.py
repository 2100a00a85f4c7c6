"""Routing by groups and orthogonalised momentum over more than 2^31 elements: rows and matrices repeat, and so have the results to."""
import pytest
import torch

from .test_gpu_muon import _bits, _gradient

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,rows,cols", [(45000, 128, 384), (45007, 384, 128), (151, 2048, 7168), (24000, 300, 301)])
def test_matrices(n, rows, cols):
    from paper_2605_23764_b200 import MoeMuon
    assert n * rows * cols > 2 ** 31
    base = _gradient(4, rows, cols, 1)
    G = torch.empty(n, rows, cols, dtype=torch.bfloat16, device="cuda")
    for i in range(4):
        G[i::4] = base[i]
    muon = MoeMuon(n, rows, cols)
    out = muon.orthogonalize(G, out=G)
    assert muon.status() == (0, 0) and out is G
    want = MoeMuon(4, rows, cols).orthogonalize(base)
    for i in range(4):
        assert bool((_bits(out[-4 + i]) == _bits(want[(n - 4 + i) % 4])).all())
        for part in _bits(out[i::4]).split(256):
            assert bool((part == _bits(out[i])).all())


@pytest.mark.parametrize("sigmoid,renorm", [(True, True), (False, False)])
def test_tokens(sigmoid, renorm):
    from paper_2605_23764_b200 import MoeLayer
    T, E, k = 2 ** 21 + 37, 1024, 2
    g = torch.Generator(device="cuda").manual_seed(0)
    base = torch.randn(64, E, device="cuda", generator=g)
    bias = torch.randint(-100, 101, (E,), device="cuda", generator=g) * 1e-4
    logits = base.repeat(T // 64 + 1, 1)[:T].contiguous()
    assert logits.numel() > 2 ** 31
    layer, few = MoeLayer(T, 64, E, k, 0, 64, renorm=renorm, sigmoid_gate=sigmoid), MoeLayer(64, 64, E, k, 0, 64, renorm=renorm, sigmoid_gate=sigmoid)
    ids, w, counts = layer.route_grouped(logits, bias, 32, 8, 2, 2.5, with_counts=True)
    rid, rw = few.route_grouped(base, bias, 32, 8, 2, 2.5)
    whole = T // 64 * 64
    assert bool((ids[:whole].view(-1, 64, k) == rid).all()) and torch.equal(ids[whole:], rid[:T - whole])
    assert bool((w[:whole].view(-1, 64, k) == rw).all()) and torch.equal(w[whole:], rw[:T - whole])
    assert torch.equal(counts.long(), torch.bincount(ids.view(-1).long(), minlength=E))
    dw = torch.randn(64, k, device="cuda", generator=g)
    d = layer.route_grouped_bwd(logits, ids, dw.repeat(T // 64 + 1, 1)[:T].contiguous(), 2.5)
    rd = few.route_grouped_bwd(base, rid, dw, 2.5)
    for part in d[:whole].view(-1, 64, E).split(4096):
        assert bool((part == rd).all())
    assert torch.equal(d[whole:], rd[:T - whole]) and layer.status() == (0, 0)
