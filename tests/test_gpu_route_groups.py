"""Routing by groups with a bias, its gradient and the bias' update against the 64-bit statement.

Tolerances.  Ids are whole numbers and equal, but for rows that two 64-bit computations may order differently (undecided(), with its
proof: sums of different scores that meet to 3e-18).  A sigmoid in fp32 is off by 3 x 2^-23 of itself (2 units of the exponential, an addition, a
division); exp(l - max) by (R + 2) 2^-23 with logits within R of one another, a softmax score by twice that and the sum's E 2^-24 / 32;
renormalising adds the sum of k terms and a division: (2 R + k + 24) 2^-23 covers all of them.  An entry of the gradient is a product of such factors
with a sum of k + 1 terms of at most `size`."""
import numpy as np
import pytest
import torch

from . import route_groups_ref as R

pytestmark = pytest.mark.gpu
U = 2.0 ** -23


def _layer(T, E, k, sigmoid=False, renorm=False):
    from paper_2605_23764_b200 import MoeLayer
    return MoeLayer(max(T, 1), 64, E, k, 0, 64, renorm=renorm, sigmoid_gate=sigmoid)


def _dev(a, t=None):
    return None if a is None else torch.as_tensor(np.ascontiguousarray(a), dtype=t).cuda()


def _spread(logits):
    fin = np.where(np.isfinite(logits), logits, 0).astype(np.float64)
    return float(fin.max() - fin.min()) if fin.size else 0.0


def _check(logits, k, bias, groups, sigmoid, renorm, layer=None, dw=None):
    T, E = logits.shape
    n_groups, top_groups, group_top, scale = groups
    layer = layer or _layer(T, E, k, sigmoid, renorm)
    l = _dev(logits)
    ids, w, counts = layer.route_grouped(l, _dev(bias), n_groups, top_groups, group_top, scale, with_counts=True)
    rng = np.random.default_rng(T + E)
    dw = rng.normal(size=(T, k)).astype(np.float32) if dw is None else dw
    d = layer.route_grouped_bwd(l, ids, _dev(dw), scale)
    torch.cuda.synchronize()
    assert layer.status() == (0, 0)
    rid, rw = R.fwd(logits, k, bias, n_groups, top_groups, group_top, scale, sigmoid, renorm)
    ids, w, counts, d = (t.cpu().numpy() for t in (ids, w, counts, d))
    # rows whose choice 64 bits do not settle go either way; the statement follows the one taken
    open_ = R.undecided(logits, bias, k, n_groups, top_groups, group_top, sigmoid)
    assert open_.sum() <= 1 + T // 8
    for t in np.flatnonzero(open_):
        c = R.scores(logits, sigmoid)[t] + (0.0 if bias is None else bias.astype(np.float64))
        best = -np.sort(-c.reshape(n_groups, -1), 1)[:, :group_top].sum(1)
        off = 2.0 ** -44 * np.abs(c).max()
        assert len(set(ids[t])) == k and np.all(best[ids[t] // (E // n_groups)] >= np.sort(best)[-top_groups] - off)
        assert np.all(np.diff((c if bias is not None else logits[t])[ids[t]]) <= off)
        rid[t], p = ids[t], R.scores(logits, sigmoid)[t, ids[t]]
        rw[t] = (p / p.sum() if renorm else p) * scale
    assert np.array_equal(ids, rid), np.argwhere((ids != rid).any(1))[:5]
    assert np.array_equal(counts, np.bincount(rid.reshape(-1), minlength=E))
    spread = _spread(logits)
    assert np.all(np.abs(w - rw) <= (2 * spread + k + 24) * U * rw + 1e-37), np.abs(w - rw).max()
    rd, size = R.bwd(logits, rid, dw, scale, sigmoid, renorm)
    assert np.all(np.abs(d - rd) <= (4 * spread + 4 * k + 64) * U * size + 1e-36), np.abs(d - rd).max()


SHAPES = [  # T, E, k, n_groups, top_groups, group_top
    (1, 1, 1, 1, 1, 1), (1, 256, 8, 8, 4, 2), (300, 256, 8, 8, 4, 2), (257, 8, 2, 2, 1, 2), (100, 160, 6, 8, 3, 1), (33, 150, 6, 10, 3, 2),
    (77, 130, 5, 1, 1, 1), (64, 64, 6, 32, 7, 2), (50, 96, 9, 3, 2, 2), (40, 512, 10, 16, 5, 2), (19, 1024, 32, 32, 9, 2), (21, 1024, 32, 4, 1, 1),
    (9, 1000, 31, 8, 2, 2), (30, 32, 32, 4, 4, 1), (31, 64, 32, 2, 1, 2), (45, 24, 3, 8, 5, 1), (200, 33, 4, 11, 6, 2)]


@pytest.mark.parametrize("T,E,k,g,top,gt", SHAPES)
@pytest.mark.parametrize("sigmoid,renorm", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("biased", [True, False])
def test_against_the_statement(T, E, k, g, top, gt, sigmoid, renorm, biased):
    rng = np.random.default_rng(T * E + k)
    logits = (rng.normal(size=(T, E)) * 1.7).astype(np.float32)
    bias = (rng.integers(-100, 101, E) * 1e-3 * (1.0 if sigmoid else 0.05)).astype(np.float32) if biased else None
    _check(logits, k, bias, (g, top, gt, 2.5), sigmoid, renorm)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("seed", range(3))
def test_near_ties_are_decided_in_64_bits(sigmoid, seed):
    """Logits one fp32 step apart, biases that undo score differences almost exactly, equal values among them."""
    rng = np.random.default_rng(seed)
    T, E, k = 200, 64, 8
    base = rng.normal(size=(T, 1)).astype(np.float32)
    logits = np.repeat(base, E, 1)
    steps = rng.integers(-2, 3, (T, E))
    for _ in range(2):
        logits = np.where(steps > 0, np.nextafter(logits, np.float32(9)), np.where(steps < 0, np.nextafter(logits, np.float32(-9)), logits)).astype(np.float32)
        steps = steps - np.sign(steps)
    bias = (rng.integers(-2, 3, E) * 2.0 ** -24).astype(np.float32)
    for groups in ((1, 1, 1, 1.0), (8, 3, 2, 1.0), (4, 2, 1, 1.0)):
        for b in (None, bias):
            _check(logits, k, b, groups, sigmoid, True)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_rows_with_infinities_and_equal_rows(sigmoid, renorm):
    rng = np.random.default_rng(5)
    T, E, k = 120, 40, 6
    logits = (rng.normal(size=(T, E))).astype(np.float32)
    logits[rng.random((T, E)) < 0.5] = -np.inf
    logits[3] = -np.inf              # nothing to choose from
    logits[4, :] = -np.inf
    logits[4, 17] = 0.25             # one expert
    logits[5] = 0.0                  # padding
    logits[7] = -100 + rng.normal(size=E)
    logits[8] = 100 + rng.normal(size=E) * 0.1
    bias = (rng.integers(-50, 51, E) * 1e-3).astype(np.float32)
    for rows in (slice(0, 7), slice(7, 8), slice(8, 9), slice(9, T)):   # rows 7 and 8 have a spread of their own
        if sigmoid and rows == slice(8, 9):
            continue                 # sigmoids of 100 are 1 in 64 bits: ties there, not in the logits
        for groups in ((5, 2, 2, 2.0), (1, 1, 1, 1.0), (10, 4, 1, 1.0)):
            part = logits[rows]
            for b in (bias, None):
                _check(part, k, b, groups, sigmoid, renorm)


def test_lowest_values_do_not_break_a_row():
    layer = _layer(4, 16, 3, True, True)
    l = torch.full((4, 16), torch.finfo(torch.float32).min, device="cuda")
    l[1, 5] = 1.0
    l[2] = float("nan")
    l[3, 3] = float("inf")
    ids, w = layer.route_grouped(l, torch.zeros(16, device="cuda"), 4, 2, 2)
    assert ids[0].tolist() == [0, 1, 2] and ids[1, 0] == 5 and ids[3, 0] == 3
    assert bool(((ids >= 0) & (ids < 16)).all()) and all(len(set(r)) == 3 for r in ids.tolist())
    assert torch.allclose(w[0].cpu(), torch.full((3,), 1 / 3)) and w[1].tolist() == [1.0, 0.0, 0.0]


@pytest.mark.parametrize("sigmoid,renorm", [(True, True), (True, False), (False, True), (False, False)])
def test_gradient_with_odd_ids_padding_and_accumulation(sigmoid, renorm):
    rng = np.random.default_rng(8)
    T, E, k = 75, 130, 6
    logits = rng.normal(size=(T, E)).astype(np.float32)
    ids = np.argsort(-logits, 1)[:, :k].astype(np.int32)
    ids[::3, 2] = ids[::3, 0]        # named twice
    ids[1::4, 1] = -1
    ids[2::5, k - 1] = E
    ids[7] = -1
    dw = rng.normal(size=(T, k)).astype(np.float32)
    dw[10:13] = 0.0
    dirty = logits.copy()
    dirty[10:13] = np.nan            # padding may hold anything where no gradient arrives
    layer = _layer(T, E, k, sigmoid, renorm)
    d = layer.route_grouped_bwd(_dev(dirty), _dev(ids), _dev(dw), 1.5)
    rd, size = R.bwd(logits, ids, dw, 1.5, sigmoid, renorm)
    tol = (4 * _spread(logits) + 4 * k + 64) * U * size + 1e-36
    assert np.all(np.abs(d.cpu().numpy() - rd) <= tol)
    assert not d[10:13].any() and not d[7].any()
    start = rng.normal(size=(T, E)).astype(np.float32)
    acc = _dev(start)
    out = layer.route_grouped_bwd(_dev(dirty), _dev(ids), _dev(dw), 1.5, d_logits=acc, accumulate=True)
    assert out is acc
    assert np.all(np.abs(acc.cpu().numpy() - (start + rd)) <= tol + 3 * U * (np.abs(start) + np.abs(rd)))
    assert np.array_equal(acc.cpu().numpy()[10:13], start[10:13])


@pytest.mark.parametrize("E", [1, 8, 33, 256, 1000, 1024])
@pytest.mark.parametrize("n_seq", [1, 7])
def test_bias_update(E, n_seq):
    rng = np.random.default_rng(E)
    counts = rng.integers(0, 50, (n_seq, E)).astype(np.int32)
    counts[:, E // 2:] = counts[:, :1] if E > 1 else counts[:, E // 2:]
    if E == 1024:
        counts[:] = 2 ** 30          # sums beyond 32 bits; all even: nothing moves
        counts[0, 3] -= 1
    bias = rng.normal(size=E).astype(np.float32)
    layer = _layer(1, E, 1)
    b, c = _dev(bias), _dev(counts if n_seq > 1 else counts[0])
    out = layer.bias_update(b, c, 1e-3, out=torch.empty_like(b))
    total = counts.astype(np.int64).sum(0)
    want = bias + np.float32(1e-3) * np.sign(total.sum() - E * total).astype(np.float32)
    assert np.array_equal(out.cpu().numpy(), want.astype(np.float32)) and np.array_equal(b.cpu().numpy(), bias)
    assert layer.bias_update(b, c, 1e-3) is b and torch.equal(b, out)


def test_many_tokens_of_every_doubt():
    """More tokens than a wave of warps, ordinary ones beside ones with ties; the counts of all."""
    rng = np.random.default_rng(1)
    T, E, k = 20000, 32, 4
    logits = rng.normal(size=(T, E)).astype(np.float32)
    logits[rng.random(T) < 0.3] = np.round(logits[rng.random(T) < 0.3][:1], 0)
    logits[::3] = np.round(logits[::3])
    bias = (rng.integers(-3, 4, E) * 0.125).astype(np.float32)
    _check(logits, k, bias, (4, 2, 2, 1.0), True, True)


def test_a_training_step_of_the_router():
    """Routing, counts without padding from the balance loss, both gradients in one tensor, the layer, the next bias."""
    from paper_2605_23764_b200 import MoeLayer
    from . import balance_ref as B
    T, d, E, k, F = 192, 128, 32, 4, 64
    g = torch.Generator().manual_seed(2)
    layer = MoeLayer(T, d, E, k, 1, F, renorm=True, sigmoid_gate=True, save_for_bwd=True)
    x = torch.randn(T, d, generator=g).to(torch.bfloat16).cuda()
    W1 = (torch.randn(E + 1, 2 * F, d, generator=g) / d ** 0.5).to(torch.bfloat16).cuda()
    W2 = (torch.randn(E + 1, d, F, generator=g) / d ** 0.5).to(torch.bfloat16).cuda()
    logits = torch.randn(T, E, generator=g).cuda()
    bias = (torch.randint(-9, 10, (E,), generator=g) * 0.01).cuda()
    mask = (torch.arange(T) % 5 != 0).to(torch.uint8).cuda()
    ids, w = layer.route_grouped(logits, bias, 4, 2, 2, 2.5)
    out = layer.ffn_fwd(x, ids, w, W1, W2)
    losses, counts, prob, tokens = layer.balance_fwd(logits, ids, token_mask=mask)
    dx, dW1, dW2, dw = layer.ffn_bwd(torch.ones_like(out), x, ids, w, W1, W2)
    dl = layer.balance_bwd(logits, ids, counts, tokens, torch.tensor([1e-2, 1e-3]).cuda(), None, token_mask=mask)
    both = layer.route_grouped_bwd(logits, ids, dw, 2.5, d_logits=dl.clone(), accumulate=True)
    new = layer.bias_update(bias, counts, 1e-3, out=torch.empty_like(bias))
    assert layer.status() == (0, 0) and torch.isfinite(dx).all()
    alone = layer.route_grouped_bwd(logits, ids, dw, 2.5)
    assert torch.equal(both, dl + alone)
    rid, _ = R.fwd(logits.cpu().numpy(), k, bias.cpu().numpy(), 4, 2, 2, 2.5, True, True)
    assert np.array_equal(ids.cpu().numpy(), rid)
    c = np.bincount(rid[mask.cpu().numpy() != 0].reshape(-1), minlength=E)
    assert np.array_equal(counts.cpu().numpy()[0], c)
    assert np.array_equal(new.cpu().numpy(), (bias.cpu().numpy() + np.float32(1e-3) * np.sign(c.sum() - E * c)).astype(np.float32))


def test_captured_and_replayed():
    T, E, k = 130, 256, 8
    layer = _layer(T, E, k, True, True)
    logits = torch.randn(T, E, device="cuda")
    bias = torch.zeros(E, device="cuda")
    dw = torch.randn(T, k, device="cuda")
    run = lambda: (lambda r: r + (layer.route_grouped_bwd(logits, r[0], dw, 2.5), layer.bias_update(bias, r[2], 1e-2)))(
        layer.route_grouped(logits, bias, 8, 4, 2, 2.5, with_counts=True))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    bias.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for seed in (1, 2):
        torch.manual_seed(seed)
        logits.normal_()
        start = bias.clone()
        graph.replay()
        torch.cuda.synchronize()
        rid, _ = R.fwd(logits.cpu().numpy(), k, start.cpu().numpy(), 8, 4, 2, 2.5, True, True)
        assert np.array_equal(got[0].cpu().numpy(), rid)
        assert np.array_equal(got[2].cpu().numpy(), np.bincount(rid.reshape(-1), minlength=E))
        assert not torch.equal(bias, start)


def test_empty_batch_and_refusals():
    from paper_2605_23764_b200 import MoeError
    layer = _layer(16, 24, 4)
    l = torch.zeros(0, 24, device="cuda")
    ids, w, counts = layer.route_grouped(l, None, 4, 2, 2, with_counts=True)
    assert ids.shape == (0, 4) and not counts.any() and layer.route_grouped_bwd(l, ids, w).shape == (0, 24)
    l = torch.zeros(16, 24, device="cuda")
    for groups in ((5, 1, 1), (0, 1, 1), (4, 5, 1), (4, 0, 1), (4, 2, 3), (4, 2, 0), (24, 3, 1), (24, 12, 2), (48, 1, 1)):
        with pytest.raises(MoeError):
            layer.route_grouped(l, None, *groups)
    with pytest.raises(MoeError):
        layer.route_grouped(l, None, scale=float("nan"))
    with pytest.raises(MoeError, match="bias"):
        layer.route_grouped(l, torch.zeros(23, device="cuda"))
    with pytest.raises(MoeError, match="bias"):
        layer.route_grouped(l, torch.zeros(24, device="cuda", dtype=torch.float64))
    with pytest.raises(MoeError, match="logits"):
        layer.route_grouped(torch.zeros(24, 16, device="cuda").t(), None)
    with pytest.raises(MoeError):
        layer.route_grouped(torch.zeros(17, 24, device="cuda"))          # more than T_max
    assert len(layer.route_grouped(l, with_counts=1)) == 3 and len(layer.route_grouped(l, None, 1, 1, 1, 2, 0)) == 2
    with pytest.raises(MoeError, match="accumulate"):
        layer.route_grouped_bwd(l, torch.zeros(16, 4, dtype=torch.int32, device="cuda"), torch.zeros(16, 4, device="cuda"), accumulate=True)
    with pytest.raises(MoeError, match="counts"):
        layer.bias_update(torch.zeros(24, device="cuda"), torch.zeros(23, dtype=torch.int32, device="cuda"), 1e-3)
    with pytest.raises(MoeError):
        layer.bias_update(torch.zeros(24, device="cuda"), torch.zeros(24, dtype=torch.int32, device="cuda"), float("inf"))
