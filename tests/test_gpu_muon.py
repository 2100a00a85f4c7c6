"""Orthogonalised momentum against plain statements in 64 bits.

Tolerances.  One step with a single coefficient has a bound for every entry, from absolute values: operands are fp16, off by at most 2^-11 of
themselves (below 2^-14 of their scaling by 2^-25 of it), and a result in bf16 by 2^-8.  a alone: X is held to 2^-22, so the result is
the rounding to bf16.  b alone: A = X X^T takes two roundings of X and its own, b A one, the product's X one: five times 2^-11 of
|X| |X^T| |X|, and fp32 sums of K terms K 2^-24 each.  c alone: two of A with three each, B's and X's: eight of |X| |X^T| |X| |X^T| |X|.

Five steps go by the norm.  A rounding's root mean square is 2^-11 / sqrt(3) of the entry; B's norm is at most 2.75 times X' / X's (0.7)
where singular values are near 1, 1.1e-3 of X' a step, A's rounding enters by |b + 2 c A| <= 4.8 at most likewise, what came in by
|f'| < 1.2 on most of 0.7 .. 1.2: three steps' worth together, 3e-3, and bf16's 2^-8 / sqrt(3) / 1.33: 5e-3 covers their sum."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
COEF = (3.4445, -4.7750, 2.0315)
NORM = 5e-3
BF16, H = 2.0 ** -8, 2.0 ** -11


def _gradient(n, rows, cols, seed, dtype=torch.bfloat16, scale=1e-4):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = max(1, min(rows, cols))
    a = torch.randn(n, rows, r, device="cuda", generator=g) * torch.arange(1, r + 1, device="cuda").rsqrt()
    return ((a @ torch.randn(n, r, cols, device="cuda", generator=g) + 0.5 * torch.randn(n, rows, cols, device="cuda", generator=g)) * scale).to(dtype)


def _exact(u, coef=COEF, steps=5, eps=1e-7):
    x = u.double()
    t = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if t else x
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + eps)
    triples = [coef] * steps if isinstance(coef[0], float) else coef
    for a, b, c in triples:
        A = x @ x.transpose(1, 2)
        x = a * x + (b * A + c * A @ A) @ x
    return x.transpose(1, 2) if t else x


def _near(got, want, norm=NORM):
    """Every matrix of its own, in the norm and entry by entry."""
    d = (got.double() - want).flatten(1)
    w = want.flatten(1)
    size = w.norm(dim=1)
    assert torch.isfinite(got).all()
    assert bool((d.norm(dim=1) <= norm * size + 1e-30).all()), (d.norm(dim=1) / size).max()
    rms = size / w.shape[1] ** 0.5
    assert bool((d.abs() <= 10 * norm * rms[:, None] + BF16 * w.abs() + 1e-30).all())


SHAPES = [(1, 1, 1), (3, 1, 8), (2, 9, 1), (4, 16, 16), (3, 28, 43), (2, 43, 28), (5, 64, 64), (16, 128, 256), (8, 256, 128), (2, 129, 257), (2, 257, 129),
          (3, 130, 1000), (3, 1000, 130), (2, 333, 517), (1, 512, 512), (1, 700, 301), (2, 384, 640), (1, 256, 2056), (1, 2056, 264), (1, 1408, 2048), (40, 72, 200),
          (2, 128, 384), (2, 384, 128), (1, 129, 384), (1, 128, 385), (1, 385, 65), (700, 24, 40), (150, 257, 260), (1, 64, 4096), (1, 3000, 136),
          (1, 8, 65536), (1, 65536, 8), (3, 20000, 130), (1, 1, 5000), (2, 5001, 1), (1, 2049, 2047)]


@pytest.mark.parametrize("n,rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_orthogonalize(n, rows, cols, dtype):
    from paper_2605_23764_b200 import MoeMuon
    G = _gradient(n, rows, cols, n + rows + cols, dtype)
    muon = MoeMuon(n, rows, cols)
    out = muon.orthogonalize(G)
    assert out.shape == G.shape and out.dtype == torch.bfloat16 and muon.status() == (0, 0)
    _near(out, _exact(G))


@pytest.mark.parametrize("n,rows,cols", [(2, 16, 24), (3, 100, 300), (3, 300, 100), (1, 257, 391), (2, 391, 257), (1, 640, 512)])
@pytest.mark.parametrize("which", [0, 1, 2])
def test_one_step_with_one_coefficient(n, rows, cols, which):
    from paper_2605_23764_b200 import MoeMuon
    coef = [0.0, 0.0, 0.0]
    coef[which] = (2.5, -1.75, 1.25)[which]
    G = _gradient(n, rows, cols, 7 + which, torch.float32)
    out = MoeMuon(n, rows, cols, coefficients=coef, steps=1, eps=0.0).orthogonalize(G)
    want = _exact(G, tuple(coef), 1, 0.0)
    x = G.double().abs()
    x = x / x.square().sum((1, 2), keepdim=True).sqrt()
    x = x.transpose(1, 2) if rows > cols else x
    m, l = min(rows, cols), max(rows, cols)
    if which == 0:
        bound = torch.full_like(x, 0.0) + 2.0 ** -21 * 2.5 * x
    elif which == 1:
        bound = (5 * H + (l + m) * 2.0 ** -24) * 1.75 * (x @ x.transpose(1, 2) @ x) + 2.0 ** -34 * x.sum(1, keepdim=True)
    else:
        A = x @ x.transpose(1, 2)
        bound = (8 * H + (l + 2 * m) * 2.0 ** -24) * 1.25 * (A @ A @ x) + 2.0 ** -34 * x.sum(1, keepdim=True)
    bound = bound.transpose(1, 2) if rows > cols else bound
    assert bool(((out.double() - want).abs() <= 1.01 * bound + BF16 * want.abs() + 1e-30).all()), ((out.double() - want).abs() / (bound + BF16 * want.abs())).max()


@pytest.mark.parametrize("coef,steps", [(COEF, 1), (COEF, 3), (COEF, 4), (COEF, 7), ((1.5, -0.5, 0.0), 12), ((1.875, -1.25, 0.375), 8),
                                        ([(4.0, -7.0, 3.5), (3.5, -5.0, 2.2), (1.875, -1.25, 0.375)], 3)])
@pytest.mark.parametrize("rows,cols", [(96, 224), (224, 96), (80, 80)])
def test_other_polynomials(coef, steps, rows, cols):
    from paper_2605_23764_b200 import MoeMuon
    G = _gradient(3, rows, cols, steps)
    _near(MoeMuon(3, rows, cols, coefficients=coef, steps=steps).orthogonalize(G), _exact(G, coef, steps))


@pytest.mark.parametrize("rows,cols", [(256, 400), (400, 256)])
@pytest.mark.parametrize("kind", ["low_rank", "one_large", "steep", "identity"])
def test_spectra(rows, cols, kind):
    """Gradients of few tokens, one direction far above the rest, values over four decades, all alike."""
    from paper_2605_23764_b200 import MoeMuon
    g = torch.Generator(device="cuda").manual_seed(3)
    m = min(rows, cols)
    a, b = torch.randn(rows, m, device="cuda", generator=g), torch.randn(m, cols, device="cuda", generator=g)
    if kind == "low_rank":
        G = a[:, :64] @ b[:64]
    elif kind == "one_large":
        G = 40 * a[:, :1] @ b[:1] + 0.1 * torch.randn(rows, cols, device="cuda", generator=g)
    elif kind == "steep":
        G = (a * torch.logspace(0, -4, m, device="cuda")) @ b
    else:
        G = torch.eye(max(rows, cols), device="cuda")[:rows, :cols]
    G = G.to(torch.bfloat16)[None].contiguous()
    _near(MoeMuon(1, rows, cols).orthogonalize(G), _exact(G))


def _noise(G):
    """What roundings relative to the largest singular value can do to the smaller ones, in the norm, once steps enough have brought all of them
    to 1: a step's 2^-11 / sqrt(3) x 2.75 of it (the norm of B) enters each, and a step later they are 3.4445 times as large, so what
    enters adds up to 3.2e-4 of the largest, 3.2e-4 / tau of a value tau times as large."""
    s = torch.linalg.svdvals(G.double())
    return (3.2e-4 / (s / s[:, :1]).clamp(min=1e-30)).clamp(max=1.0).square().mean(1).sqrt().max().item()


@pytest.mark.parametrize("n,rows,cols,steps", [(50, 300, 700, 5), (50, 700, 300, 5), (150, 200, 440, 6), (50, 264, 1056, 7), (150, 130, 401, 5), (25, 520, 1200, 9)])
@pytest.mark.parametrize("kind", ["full", "low_rank"])
def test_many_matrices_and_steps(n, rows, cols, steps, kind):
    """More tiles than pairs of SMs, five steps and more.  Gradients of fewer tokens than either side has, whose other singular values are what
    bf16 makes of zero, 1e-3 of the largest, are brought to 1 by more than five steps: there what roundings do to those counts (_noise)."""
    from paper_2605_23764_b200 import MoeMuon
    G = _gradient(n, rows, cols, steps)
    norm = NORM
    if kind == "low_rank":
        g = torch.Generator(device="cuda").manual_seed(9)
        G = (torch.randn(n, rows, 100, device="cuda", generator=g) @ torch.randn(n, 100, cols, device="cuda", generator=g)).to(torch.bfloat16)
        if steps > 5:
            norm += _noise(G[:2])
    muon = MoeMuon(n, rows, cols, steps=steps)
    out = muon.orthogonalize(G)
    assert muon.status() == (0, 0)
    _near(out, _exact(G, steps=steps), norm)
    W, M = _gradient(n, rows, cols, 1, scale=0.1), torch.zeros(n, rows, cols, device="cuda")
    W1, _ = muon.step(W, M, G, lr=0.01, W_out=torch.empty_like(W), M_out=torch.empty_like(M))
    x = _exact(1.95 * G.double(), steps=steps)
    want = W.double() - 0.01 * x
    assert bool(((W1.double() - want).abs() <= 0.01 * 10 * norm * x.abs().amax() + BF16 * (want.abs() + 0.01 * x.abs())).all())


def _bits(t):
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


@pytest.mark.parametrize("rows,cols", [(64, 136), (136, 64), (100, 51)])
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


@pytest.mark.parametrize("n,rows,cols", [(3, 96, 160), (2, 160, 96), (2, 130, 75), (1, 1, 7)])
@pytest.mark.parametrize("nesterov", [True, False])
def test_step(n, rows, cols, nesterov):
    from paper_2605_23764_b200 import MoeMuon
    g = torch.Generator(device="cuda").manual_seed(rows)
    W = (torch.randn(n, rows, cols, device="cuda", generator=g) * 0.1).to(torch.bfloat16)
    dW, M = _gradient(n, rows, cols, 5), _gradient(n, rows, cols, 6, torch.float32, 1e-3)
    mu, lr, wd, scale = np.float32(0.9), np.float32(0.02), np.float32(0.1), np.float32(1.5)
    muon = MoeMuon(n, rows, cols, momentum=0.9, nesterov=nesterov)
    W1, M1 = muon.step(W, M, dW, lr=0.02, weight_decay=0.1, scale=1.5, W_out=torch.empty_like(W), M_out=torch.empty_like(M))
    m = float(mu) * M.double() + dW.double()
    assert bool(((M1.double() - m).abs() <= 2.0 ** -24 * m.abs() + 1e-44).all())
    x = _exact(dW.double() + float(mu) * m if nesterov else m)
    rate = float(lr) * float(scale)
    want = (1 - float(lr) * float(wd)) * W.double() - rate * x
    rms = x.flatten(1).norm(dim=1) / (rows * cols) ** 0.5
    # the update is off as X is, without X's own rounding to bf16; the result rounds to bf16; three fp32 roundings
    assert bool(((W1.double() - want).abs() <= rate * 10 * NORM * rms[:, None, None] + (BF16 + 3 * 2.0 ** -24) * (want.abs() + rate * x.abs())).all())
    W2, M2 = W.clone(), M.clone()
    got = muon.step(W2, M2, dW, lr=0.02, weight_decay=0.1, scale=1.5)
    assert got[0] is W2 and got[1] is M2 and torch.equal(_bits(W2), _bits(W1)) and torch.equal(_bits(M2), _bits(M1))
    assert muon.status() == (0, 0)


@pytest.mark.parametrize("n,rows,cols", [(2, 72, 136), (2, 136, 72)])
def test_unaligned_tensors_give_the_same_bits(n, rows, cols):
    from paper_2605_23764_b200 import MoeMuon
    muon = MoeMuon(n, rows, cols)

    def shifted(t):
        s = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape)
        return s.copy_(t)
    W = (_gradient(n, rows, cols, 4, scale=0.1))
    dW, M = _gradient(n, rows, cols, 5), _gradient(n, rows, cols, 6, torch.float32)
    a = muon.step(W, M, dW, 0.02, W_out=torch.empty_like(W), M_out=torch.empty_like(M))
    b = muon.step(shifted(W), shifted(M), shifted(dW), 0.02, W_out=shifted(W), M_out=shifted(M))
    assert b[0].data_ptr() % 16 and torch.equal(_bits(a[0]), _bits(b[0])) and torch.equal(_bits(a[1]), _bits(b[1]))
    assert torch.equal(_bits(muon.orthogonalize(dW)), _bits(muon.orthogonalize(shifted(dW), out=shifted(W))))


def test_more_matrices_than_the_workspace_holds():
    """A batch that goes through the workspace in turns gives each matrix what it gets alone; outputs have no room behind them."""
    from paper_2605_23764_b200 import MoeMuon
    n, rows, cols = 70, 1024, 1536
    G = _gradient(n, rows, cols, 2)
    muon = MoeMuon(n, rows, cols)
    assert muon.workspace.numel() < 2 ** 30 + 2 ** 20
    room = torch.full((n * rows * cols + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = room[:n * rows * cols].view(n, rows, cols)
    muon.orthogonalize(G, out=out)
    assert muon.launches() > 3 and bool((room[-64:] == 7).all())
    one = MoeMuon(1, rows, cols)
    for i in (0, 33, 34, 46, 47, 69):
        assert torch.equal(_bits(out[i]), _bits(one.orthogonalize(G[i:i + 1])[0])), i
    _near(out[68:], _exact(G[68:]))


def test_two_handles_on_two_streams():
    from paper_2605_23764_b200 import MoeMuon
    Ga, Gb = _gradient(5, 200, 264, 1), _gradient(4, 300, 136, 2)
    a, b = MoeMuon(5, 200, 264), MoeMuon(4, 300, 136)
    want = a.orthogonalize(Ga), b.orthogonalize(Gb)
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(s):
            x = a.orthogonalize(Ga)
        with torch.cuda.stream(t):
            y = b.orthogonalize(Gb)
        torch.cuda.synchronize()
        assert torch.equal(_bits(x), _bits(want[0])) and torch.equal(_bits(y), _bits(want[1]))


def test_captured_and_replayed():
    from paper_2605_23764_b200 import MoeMuon
    W, M, dW = _gradient(3, 96, 168, 1, scale=0.1), _gradient(3, 96, 168, 2, torch.float32), _gradient(3, 96, 168, 3)
    muon = MoeMuon(3, 96, 168)
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
    torch.cuda.synchronize()
    assert torch.equal(_bits(Wg), _bits(We)) and torch.equal(_bits(Mg), _bits(Me))


def test_a_layers_training_step():
    """Forward, backward and the update of both weight tensors, as they lie; experts without tokens keep their weights but for the decay."""
    from paper_2605_23764_b200 import MoeLayer, MoeMuon
    T, d, E, k, S, F = 64, 128, 12, 2, 1, 64
    g = torch.Generator().manual_seed(4)
    layer = MoeLayer(T, d, E, k, S, F, renorm=True, save_for_bwd=True)
    x = torch.randn(T, d, generator=g).to(torch.bfloat16).cuda()
    W1 = (torch.randn(E + S, 2 * F, d, generator=g) / d ** 0.5).to(torch.bfloat16).cuda()
    W2 = (torch.randn(E + S, d, F, generator=g) / d ** 0.5).to(torch.bfloat16).cuda()
    logits = torch.randn(T, E, generator=g).cuda()
    logits[:, 5] = -float("inf")
    up, down = MoeMuon.for_gate_up(layer), MoeMuon.for_down(layer)
    M1, M2 = torch.zeros(W1.shape, device="cuda"), torch.zeros(W2.shape, device="cuda")
    for _ in range(2):
        ids, w = layer.route_grouped(logits, torch.zeros(E, device="cuda"), 4, 2, 2)
        out = layer.ffn_fwd(x, ids, w, W1, W2)
        dx, dW1, dW2, dw = layer.ffn_bwd(out, x, ids, w, W1, W2)
        old1, old2, m1 = W1.clone(), W2.clone(), M1.double()
        up.step(W1, M1, dW1, lr=0.01, scale=0.5)
        down.step(W2, M2, dW2, lr=0.01, scale=0.5)
        assert layer.status() == (0, 0) and up.status() == (0, 0) and down.status() == (0, 0)
        assert torch.equal(W1[5], old1[5]) and torch.equal(W2[5], old2[5]) and not dW1[5].any()
        m = 0.95 * m1 + dW1.double()
        x_ = _exact((dW1.double() + 0.95 * m).view(2 * (E + S), F, d)).view(W1.shape)
        want = old1.double() - 0.005 * x_
        assert bool(((W1.double() - want).abs() <= 0.005 * 10 * NORM * x_.abs().amax() + BF16 * (want.abs() + 0.005 * x_.abs())).all())
        assert not torch.equal(W2[0], old2[0])


def test_refusals():
    from paper_2605_23764_b200 import MoeError, MoeMuon, binding
    for bad in ((0, 8, 8), (1, 0, 8), (1, 8, 0), (1, 65537, 8), (70000, 8, 8)):
        with pytest.raises(MoeError):
            MoeMuon(*bad)
    with pytest.raises(MoeError):
        MoeMuon(1, 8, 8, eps=-1.0)
    muon = MoeMuon(2, 16, 24)
    G = torch.zeros(2, 16, 24, dtype=torch.bfloat16, device="cuda")
    f = torch.zeros(2, 16, 24, device="cuda")
    with pytest.raises(MoeError, match="G"):
        muon.orthogonalize(G[:1])
    with pytest.raises(MoeError, match="G"):
        muon.orthogonalize(G.half())
    with pytest.raises(MoeError, match="G"):
        muon.orthogonalize(torch.zeros(2, 24, 16, dtype=torch.bfloat16, device="cuda").transpose(1, 2))
    with pytest.raises(MoeError, match="M"):
        muon.step(G, G, G, 0.1)
    with pytest.raises(MoeError, match="dW"):
        muon.step(G, f, f, 0.1)
    with pytest.raises(MoeError, match="W_out"):
        muon.step(G, f, G, 0.1, W_out=G[:1])
    for bad in (dict(lr=float("nan")), dict(lr=0.1, weight_decay=float("inf")), dict(lr=0.1, scale=float("nan"))):
        with pytest.raises(MoeError):
            muon.step(G, f, G, **bad)
    keep = [binding.moe_muon_step(muon.handle, G, f, G, 0.9, n, 0.1, 0.0, 1.0, torch.empty_like(G), torch.empty_like(f)) for n in (1, True, 0, False)]
    assert keep == [None] * 4
    muon.close()
    with pytest.raises(MoeError, match="unknown muon handle"):
        muon.orthogonalize(G)
    shape = binding.moe_muon_shape(2, 16, 24, COEF, 5, 1e-7)
    with pytest.raises(MoeError):   # too small a workspace
        binding.moe_muon_create(shape, torch.empty(binding.moe_muon_workspace_bytes(shape) - 1, dtype=torch.uint8, device="cuda"))
    h = binding.moe_muon_create(shape)   # one of its own
    out = torch.empty_like(G)
    binding.moe_muon_orthogonalize(h, G, out)
    torch.cuda.synchronize()
    assert not out.any()
    binding.moe_muon_destroy(h)


def test_a_handle_serves_streams_in_turn_and_a_capture_beside_eager_calls():
    """One handle on several streams, each waiting for the other; a graph captured from it between eager calls; memory of one's own."""
    from paper_2605_23764_b200 import MoeMuon, binding
    n, rows, cols = 6, 300, 520
    G, H = _gradient(n, rows, cols, 1), _gradient(n, rows, cols, 2)
    muon = MoeMuon(n, rows, cols)
    want = muon.orthogonalize(G), muon.orthogonalize(H)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    a.wait_stream(torch.cuda.current_stream())
    for i in range(6):
        s, t = (a, b) if i % 2 == 0 else (b, a)
        with torch.cuda.stream(s):
            outs.append(muon.orthogonalize(G if i % 3 else H))
        t.wait_stream(s)
    torch.cuda.synchronize()
    assert all(torch.equal(_bits(o), _bits(want[0] if i % 3 else want[1])) for i, o in enumerate(outs))
    out = torch.empty_like(G)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        muon.orthogonalize(G, out=out)
    eager = muon.orthogonalize(H)
    graph.replay()
    again = muon.orthogonalize(H)
    torch.cuda.synchronize()
    assert torch.equal(_bits(out), _bits(want[0])) and torch.equal(_bits(eager), _bits(want[1])) and torch.equal(_bits(again), _bits(want[1]))
    h = binding.moe_muon_create(binding.moe_muon_shape(n, rows, cols, COEF, 5, 1e-7))   # the library's own workspace
    binding.moe_muon_orthogonalize(h, G, out.zero_())
    assert binding.moe_muon_get_status(h) == (0, 0) and binding.moe_muon_last_launch_count(h) == 3
    assert torch.equal(_bits(out), _bits(want[0]))
    binding.moe_muon_destroy(h)
    G2 = G.clone()   # in its own place
    muon.orthogonalize(G2, out=G2)
    assert torch.equal(_bits(G2), _bits(want[0]))
