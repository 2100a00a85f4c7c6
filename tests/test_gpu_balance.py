"""Balance losses of the router and the whole gradient of its logits against the 64-bit statement.

Tolerances.  With logits within R of one another, exp(l - max) in fp32 is off by at most (R + 2) 2^-23 relative (the argument's two
roundings, two units of the approximation), a probability by twice that and the sum's E 2^-24 / 32: (2 R + 16) 2^-23 covers it for
E <= 1024.  A mean of n positive terms adds n 2^-24 at most.  Counts and tokens are whole numbers."""
import numpy as np
import pytest
import torch

from . import balance_ref as R

pytestmark = pytest.mark.gpu
U = 2.0 ** -23


def _case(T, E, k, seed, spread=1.5, dup=False, bad=False):
    rng = np.random.default_rng(seed)
    logits = (rng.normal(size=(T, E)) * spread).astype(np.float32)
    ids = np.argsort(-logits, 1, kind="stable")[:, :k].astype(np.int32).reshape(T, k)
    if dup and T > 2 and k > 1:
        ids[::3, 1] = ids[::3, 0]
    if bad and T > 3:
        ids[1::4, 0] = -1
        ids[2::5, k - 1] = E
    return logits, ids, (rng.normal(size=(T, k))).astype(np.float32)


def _run(logits, ids, dw, off=None, mask=None, renorm=False, sigmoid=False, dl=(0.02, 0.003), layer=None):
    from paper_2605_23764_b200 import MoeLayer
    T, E = logits.shape
    k = ids.shape[1]
    own = layer is None
    layer = layer or MoeLayer(max(T, 1), 64, E, k, 0, 64, renorm=renorm, sigmoid_gate=sigmoid)
    dev = lambda a, t=None: None if a is None else torch.as_tensor(np.ascontiguousarray(a), dtype=t).cuda()
    l, i, o, m = dev(logits), dev(ids), dev(off, torch.int32), dev(mask, torch.uint8)
    losses, counts, prob, tokens = layer.balance_fwd(l, i, o, m)
    d = layer.balance_bwd(l, i, counts, tokens, torch.tensor(dl, dtype=torch.float32).cuda(), dev(dw), o, m)
    torch.cuda.synchronize()
    assert layer.status() == (0, 0)
    if own:
        layer.close()
    return [t.cpu().numpy() for t in (losses, counts, prob, tokens, d)]


def _check(got, logits, ids, dw, off=None, mask=None, renorm=False, sigmoid=False, dl=(0.02, 0.003)):
    losses, counts, prob, tokens, d = got
    rl, rc, rp, rt = R.fwd(logits, ids, off, mask, sigmoid)
    assert np.array_equal(counts, rc) and np.array_equal(tokens, rt)
    fin = np.where(np.isfinite(logits), logits, 0).astype(np.float64)
    spread = float(fin.max() - fin.min()) if fin.size else 0.0
    rel = (2 * spread + 16) * U + max(int(rt[:-1].max(initial=0)), 1) * U / 2
    assert np.all(np.abs(prob - rp) <= rel * rp + 1e-30), np.abs(prob - rp).max()
    assert abs(losses[0] - rl[0]) <= (rel + 8 * U) * rl[0] + 1e-30, (losses, rl)
    lse = np.abs(R.rows(logits, sigmoid)[3]).max(initial=0.0)
    # logsumexp is off by the sum's relative error and its own rounding, its square by twice that times itself
    off_lse = (2 * spread + 16) * U + lse * U
    assert abs(losses[1] - rl[1]) <= 2 * lse * off_lse + (len(logits) + 8) * U * rl[1], (losses, rl)
    rd, size = R.bwd(logits, ids, rc, rt, dl, dw, off, mask, sigmoid, renorm)
    # every entry is a sum of a few products of a probability with something no larger than `size`
    assert np.all(np.abs(d - rd) <= (4 * spread + 48) * U * size[:, None] + 1e-30), np.abs(d - rd).max()


SHAPES = [(1, 4, 1), (1, 256, 8), (2, 5, 5), (7, 8, 2), (300, 8, 8), (33, 12, 3), (64, 16, 1), (130, 24, 6), (97, 33, 4), (50, 64, 6),
          (1000, 100, 8), (257, 128, 8), (77, 130, 6), (2049, 256, 8), (65, 321, 2), (40, 512, 8), (19, 1000, 32), (20, 1023, 3), (9, 1024, 8)]


@pytest.mark.parametrize("T,E,k", SHAPES)
@pytest.mark.parametrize("sigmoid,renorm", [(False, True), (True, False)])
def test_one_sequence(T, E, k, sigmoid, renorm):
    logits, ids, dw = _case(T, E, k, T + E + k, dup=True)
    opt = dict(renorm=renorm, sigmoid=sigmoid)
    _check(_run(logits, ids, dw, **opt), logits, ids, dw, **opt)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("T,E,k,n", [(2000, 256, 8, 7), (700, 130, 6, 3), (515, 8, 2, 40), (64, 64, 6, 64), (1500, 48, 4, 1100), (900, 512, 4, 5)])
def test_sequences_masks_and_odd_ids(T, E, k, n, sigmoid, renorm):
    """Uneven and empty sequences, tokens outside of them, padding, sequences that are all padding, ids named twice and out of range."""
    logits, ids, dw = _case(T, E, k, 11 * T + n, dup=True, bad=True)
    rng = np.random.default_rng(n)
    off = np.sort(rng.integers(T // 50, T - T // 40, size=n + 1)).astype(np.int32)
    mask = (rng.random(T) > 0.25).astype(np.uint8)
    mask[off[n // 2]:off[n // 2 + 1]] = 0
    opt = dict(off=off, mask=mask, renorm=renorm, sigmoid=sigmoid)
    _check(_run(logits, ids, dw, **opt), logits, ids, dw, **opt)


@pytest.mark.parametrize("T,E,k,n", [(40000, 64, 2, 1), (30000, 256, 4, 6), (9000, 1024, 8, 2)])
def test_sequences_over_many_blocks(T, E, k, n):
    from paper_2605_23764_b200 import MoeLayer
    rng = np.random.default_rng(T)
    logits = torch.from_numpy((rng.normal(size=(T, E))).astype(np.float32)).cuda()
    ids = torch.topk(logits, k, dim=1).indices.to(torch.int32).contiguous()
    off = [0] + sorted(int(v) for v in rng.integers(0, T, size=n - 1)) + [T]
    layer = MoeLayer(T, 64, E, k, 0, 64)
    losses, counts, prob, tokens = layer.balance_fwd(logits, ids, torch.tensor(off, dtype=torch.int32).cuda() if n > 1 else None)
    again = layer.balance_fwd(logits, ids, torch.tensor(off, dtype=torch.int32).cuda() if n > 1 else None)
    p = torch.softmax(logits.double(), 1)
    balance = 0.0
    for s, (a, b) in enumerate(zip(off[:-1], off[1:])):
        c = torch.bincount(ids[a:b].reshape(-1).long(), minlength=E)
        assert torch.equal(counts[s].long(), c) and int(tokens[s]) == b - a
        if b > a:
            mean = p[a:b].mean(0)
            balance += E / (k * (b - a)) * float((c * mean).sum()) / n
            # a warp adds up at most T / (4 x 148) + 32 terms, the rest are sums of a few hundred
            assert float(((prob[s] - mean).abs() / mean).max()) <= (2 * 12 + 16) * U + 600 * U
    assert abs(float(losses[0]) - balance) <= 1e-4 * balance
    lse = torch.logsumexp(logits.double(), 1)
    assert abs(float(losses[1]) - float((lse ** 2).mean())) <= 1e-5 * float((lse ** 2).mean())
    for x, y in zip((losses, counts, prob, tokens), again):
        assert torch.equal(x, y)   # the sums' order is fixed
    layer.close()


def test_masked_logits_and_rows_without_a_finite_logit():
    logits, ids, dw = _case(60, 40, 4, 5)
    logits[:, 7] = -np.inf
    logits[3::4, 20:] = -np.inf
    logits[5] = -np.inf
    logits[9] = np.finfo(np.float32).min
    ids = np.argsort(-logits, 1, kind="stable")[:, :4].astype(np.int32)
    for sigmoid in (False, True):
        for renorm in (False, True):
            got = _run(logits, ids, dw, renorm=renorm, sigmoid=sigmoid)
            assert all(np.isfinite(g).all() for g in got[2:])
            keep = np.arange(60) != 9     # (its logsumexp squared is beyond fp32)
            m = keep.astype(np.uint8)
            got = _run(logits, ids, dw, mask=m, renorm=renorm, sigmoid=sigmoid)
            clean = np.where(np.isfinite(logits) & (logits > -1e30), logits, -1e4).astype(np.float32)
            clean[5] = -np.inf
            losses, counts, prob, tokens, d = got
            rl, rc, rp, rt = R.fwd(clean, ids, None, m, sigmoid)
            assert np.array_equal(counts, rc) and np.array_equal(tokens, rt)
            np.testing.assert_allclose(prob, rp, atol=2e-6)
            np.testing.assert_allclose(losses, rl, rtol=1e-5)
            rd, size = R.bwd(clean, ids, rc, rt, (0.02, 0.003), dw, None, m, sigmoid, renorm)
            assert np.all(np.abs(d - rd)[keep] <= 100 * U * size[keep, None] + 1e-30)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("E", [6, 64, 321])
def test_one_renormalised_score_has_no_gradient(E, sigmoid):
    """w = v / v: what arrives for it leaves nothing beside the losses' gradient, which is smaller by the number of tokens."""
    T = 4000
    logits, ids, dw = _case(T, E, 1, E)
    got = _run(logits, ids, dw, renorm=True, sigmoid=sigmoid)
    alone = _run(logits, ids, None, renorm=True, sigmoid=sigmoid)
    assert np.array_equal(got[4], alone[4])
    _check(alone, logits, ids, None, renorm=True, sigmoid=sigmoid)
    # and of scores whose gradients are alike but for little, the little counts
    logits, ids, dw = _case(64, E, 3, E + 1)
    dw = (1.0 + np.round(dw * 256) * 2.0 ** -16).astype(np.float32)   # differences are exact
    got = _run(logits, ids, dw, renorm=True, sigmoid=sigmoid, dl=(0.0, 0.0))
    _check(got, logits, ids, dw - np.float32(1), renorm=True, sigmoid=sigmoid, dl=(0.0, 0.0))


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("E", [40, 41])
def test_padding_holds_anything(E, sigmoid):
    """NaN and infinities in tokens that are masked or outside of the sequences, and ids that are none."""
    T, k = 90, 4
    logits, ids, dw = _case(T, E, k, 15)
    mask = np.ones(T, np.uint8)
    mask[5:17] = 0
    off = np.array([3, 40, 80], np.int32)
    idle = (mask == 0) | (np.arange(T) < 3) | (np.arange(T) >= 80)
    clean = [g.copy() for g in _run(logits, ids, None, off, mask, sigmoid=sigmoid)]
    _check(clean, logits, ids, None, off, mask, sigmoid=sigmoid)
    for v in (np.nan, np.inf, -np.inf):
        logits[idle], ids[idle] = v, 12345678
        logits[7, ::2] = 1.0
        for want, got in zip(clean, _run(logits, ids, None, off, mask, sigmoid=sigmoid)):
            assert np.array_equal(want, got)
    assert not clean[4][idle].any()


def test_sigmoids_that_underflow_keep_their_proportions():
    logits, ids, dw = _case(50, 16, 2, 6)
    logits -= 200.0
    got = _run(logits, ids, dw, sigmoid=True, dl=(0.02, 0.0))
    _, _, rp, _ = R.fwd(logits, ids, sigmoid=True)
    # the argument l - max has 2^-16 of rounding at 200: l itself is given to that
    np.testing.assert_allclose(got[2], rp, rtol=(2 * 12 + 16 + 50) * U)
    assert np.isfinite(got[4]).all()


def test_no_tokens():
    from paper_2605_23764_b200 import MoeLayer
    layer = MoeLayer(4, 64, 8, 2, 0, 64)
    e = torch.empty
    losses, counts, prob, tokens = layer.balance_fwd(e(0, 8).cuda(), e(0, 2, dtype=torch.int32).cuda(), torch.zeros(4, dtype=torch.int32).cuda())
    assert losses.tolist() == [0.0, 0.0] and counts.shape == (3, 8) and not counts.any() and not prob.any() and not tokens.any()
    d = layer.balance_bwd(e(0, 8).cuda(), e(0, 2, dtype=torch.int32).cuda(), counts, tokens, losses, seq_offsets=torch.zeros(4, dtype=torch.int32).cuda())
    assert d.shape == (0, 8)
    layer.close()


def test_gradient_in_place_and_without_scores():
    from paper_2605_23764_b200 import MoeLayer
    T, E, k = 333, 96, 4
    logits, ids, dw = _case(T, E, k, 12)
    layer = MoeLayer(T, 64, E, k, 0, 64, renorm=True)
    l, i, g = torch.from_numpy(logits).cuda(), torch.from_numpy(ids).cuda(), torch.from_numpy(dw).cuda()
    dl = torch.tensor([0.02, 0.003]).cuda()
    _, counts, _, tokens = layer.balance_fwd(l, i)
    want = layer.balance_bwd(l, i, counts, tokens, dl, g)
    got = layer.balance_bwd(l.clone(), i, counts, tokens, dl, g)
    here = l.clone()
    layer.balance_bwd(here, i, counts, tokens, dl, g, d_logits=here)
    assert torch.equal(want, got) and torch.equal(want, here)
    alone = layer.balance_bwd(l, None, counts, tokens, dl)
    rd, size = R.bwd(logits, ids, counts.cpu().numpy(), tokens.cpu().numpy(), (0.02, 0.003))
    assert np.all(np.abs(alone.cpu().numpy() - rd) <= (4 * 12 + 48) * U * size[:, None])
    layer.close()


def test_rows_that_are_not_vectors():
    """Logits that begin at an odd element: rows of whole vectors at a place that is none."""
    from paper_2605_23764_b200 import MoeLayer
    T, E, k = 100, 64, 6
    logits, ids, dw = _case(T, E, k, 13)
    layer = MoeLayer(T, 64, E, k, 0, 64)
    l, i = torch.from_numpy(logits).cuda(), torch.from_numpy(ids).cuda()
    odd = torch.empty(T * E + 1, device="cuda")[1:].view(T, E)
    odd.copy_(l)
    a, b = layer.balance_fwd(l, i), layer.balance_fwd(odd, i)
    assert torch.equal(a[1], b[1])
    np.testing.assert_allclose(a[2].cpu().numpy(), b[2].cpu().numpy(), rtol=200 * U)
    layer.close()


def test_graphs_streams_and_a_bad_call_in_between():
    from paper_2605_23764_b200 import MoeLayer
    T, E, k = 5000, 64, 2
    logits, ids, dw = _case(T, E, k, 21)
    layer = MoeLayer(T, 64, E, k, 0, 64)
    l, i, g = torch.from_numpy(logits).cuda(), torch.from_numpy(ids).cuda(), torch.from_numpy(dw).cuda()
    off = torch.tensor([0, 1200, 1200, 4100, T], dtype=torch.int32).cuda()
    dl = torch.tensor([0.02, 0.003]).cuda()

    def step():
        losses, counts, prob, tokens = layer.balance_fwd(l, i, off)
        return losses, counts, prob, tokens, layer.balance_bwd(l, i, counts, tokens, dl, g, off)

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))
    # offsets that do not ascend give unspecified values, and the next call its own
    layer.balance_fwd(l, i, torch.tensor([4000, 100, 9000, -5, 50], dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, step()))
    layer.close()


def test_router_losses_and_layer_as_a_training_step():
    """Router, balance losses, layer and both backward calls in a row; the logits' gradient is the scores' plus the losses'."""
    from paper_2605_23764_b200 import MoeLayer, binding as B
    T, d, E, k, F = 512, 256, 32, 4, 128
    g = torch.Generator().manual_seed(9)
    x = torch.randn(T, d, generator=g).to(torch.bfloat16).cuda()
    W_r = (torch.randn(E, d, generator=g) * 0.06).to(torch.bfloat16).cuda()
    W1 = (torch.randn(E, 2 * F, d, generator=g) / d ** 0.5).to(torch.bfloat16).cuda()
    W2 = (torch.randn(E, d, F, generator=g) / F ** 0.5).to(torch.bfloat16).cuda()
    dout = torch.randn(T, d, generator=g).to(torch.bfloat16).cuda()
    layer = MoeLayer(T, d, E, k, 0, F, renorm=True, save_for_bwd=True)
    ids, w = torch.empty(T, k, dtype=torch.int32).cuda(), torch.empty(T, k).cuda()
    logits, named = torch.empty(T, E).cuda(), torch.empty(E, dtype=torch.int32).cuda()
    B.moe_router_fwd(layer.ctx, x, W_r, T, ids, w, logits, named)
    out = layer.ffn_fwd(x, ids, w, W1, W2)
    losses, counts, prob, tokens = layer.balance_fwd(logits, ids)   # between forward and backward: the saved forward stays
    assert torch.equal(counts[0], named)
    _, _, _, d_w = layer.ffn_bwd(dout, x, ids, w, W1, W2)
    dl = torch.tensor([0.01, 0.001]).cuda()
    d_logits = layer.balance_bwd(logits, ids, counts, tokens, dl, d_w)
    scores = torch.empty(T, E).cuda()
    B.moe_router_bwd(layer.ctx, logits, ids, d_w, T, scores)
    alone = layer.balance_bwd(logits, ids, counts, tokens, dl)
    assert layer.status() == (0, 0)
    size = d_w.abs().sum(1, keepdim=True) + alone.abs().max()
    assert bool(((d_logits - scores - alone).abs() <= 200 * U * size).all())
    rl, rc, rp, _ = R.fwd(logits.cpu().numpy(), ids.cpu().numpy())
    np.testing.assert_allclose(losses.cpu().numpy(), rl, rtol=1e-4)
    assert float(out.float().abs().max()) > 0
    layer.close()


def test_refusals():
    from paper_2605_23764_b200 import MoeError, MoeLayer
    layer = MoeLayer(16, 64, 8, 2, 0, 64)
    l, i = torch.zeros(16, 8).cuda(), torch.zeros(16, 2, dtype=torch.int32).cuda()
    with pytest.raises(MoeError, match="contiguous"):
        layer.balance_fwd(torch.zeros(8, 16).cuda().t(), i)
    with pytest.raises(MoeError, match="token_mask"):
        layer.balance_fwd(l, i, token_mask=torch.ones(15, dtype=torch.uint8).cuda())
    with pytest.raises(MoeError, match="token_mask"):
        layer.balance_fwd(l, i, token_mask=torch.ones(16, dtype=torch.bool).cuda())
    with pytest.raises(MoeError):
        layer.balance_fwd(l, i, seq_offsets=torch.zeros(1, dtype=torch.int32).cuda())   # no sequence
    with pytest.raises(MoeError):
        layer.balance_fwd(torch.zeros(17, 8).cuda(), torch.zeros(17, 2, dtype=torch.int32).cuda())   # more than T_max
    with pytest.raises(MoeError, match="topk_ids"):
        layer.balance_fwd(l, i[:15].clone())
    losses, counts, prob, tokens = layer.balance_fwd(l, i)
    with pytest.raises(MoeError, match="counts"):
        layer.balance_bwd(l, i, counts[:, :7].contiguous(), tokens, losses)
    with pytest.raises(MoeError, match="topk_ids|invalid"):
        layer.balance_bwd(l, None, counts, tokens, losses, torch.zeros(16, 2).cuda())
    layer.close()
