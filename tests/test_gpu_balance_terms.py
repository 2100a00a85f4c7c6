"""The gradient of the balance losses, each loss by itself and both beside the scores' at a size of their own.

Tolerances, entry by entry.  R = the row's spread + its largest size: a probability is off by e = (2 R + 16) 2^-23 relative (the
approximate exponential's argument and its two units, a quotient, a sum; sigmoids have their own exponential, hence the size).

  balance: p_i (x_i - sum p x) (1 - sig_i) -- p_i by e, x by its four roundings, sum p x by e + 4 roundings of the largest x, 1 - sig_i by a
           rounding of 1: together p_i max|x| (3 e + 16 2^-23)
  z:       2 / N lse soft_i -- soft_i by e of lse, lse by e + 2^-23 |lse|: soft_i 2 / N (|lse| (e + 8 2^-23) + e)
  scores:  as the gradient's other tests, relative to what arrives for the row."""
import numpy as np
import pytest
import torch

from . import balance_ref as R
from .test_gpu_balance import SHAPES, _case, _run

pytestmark = pytest.mark.gpu
U = 2.0 ** -23


def _bounds(logits, ids, counts, tokens, dl, off, mask, sigmoid):
    """of the balance loss's gradient and the z loss's"""
    T, E = logits.shape
    k = ids.shape[1]
    p, soft, _, lse = R.rows(logits, sigmoid)
    l = logits.astype(np.float64)
    e = (2 * (l.max(1) - l.min(1) + np.abs(l).max(1)) + 16) * U
    bal, z = np.zeros((T, E)), np.zeros((T, E))
    seqs = R.sequences(T, off, mask)
    for s, ts in enumerate(seqs):
        if len(ts):
            most = abs(dl[0]) * E / (k * len(seqs)) / len(ts) ** 2 * counts[s].max(initial=0)
            bal[ts] = p[ts] * most * (3 * e[ts] + 16 * U)[:, None]
            z[ts] = soft[ts] * (2 * abs(dl[1]) / tokens[-1] * (np.abs(lse[ts]) * (e[ts] + 8 * U) + e[ts]))[:, None]
    return bal, z


def _check_terms(logits, ids, dw, off=None, mask=None, sigmoid=False, renorm=False):
    T, E = logits.shape
    k = ids.shape[1]
    _, counts, _, tokens = R.fwd(logits, ids, off, mask, sigmoid)
    opt = dict(off=off, mask=mask, renorm=renorm, sigmoid=sigmoid)
    ref = dict(seq_offsets=off, token_mask=mask, sigmoid=sigmoid, renorm=renorm)
    grads = {}
    for dl in ((float(T), 0.0), (0.0, float(T)), (0.5 * T, -0.25 * T)):
        want, _ = R.bwd(logits, ids, counts, tokens, dl, None, **ref)
        bal, z = _bounds(logits, ids, counts, tokens, dl, off, mask, sigmoid)
        got = _run(logits, ids, None, dl=dl, **opt)[4]
        assert np.all(np.abs(got - want) <= bal + z + 1e-30), (dl, np.abs(got - want).max())
        grads[dl] = want
        # a gradient without the term would not do (k = E: every expert is named alike, and the balance loss has none)
        for term in (0, 1):
            if dl[term] and (term or k < E):
                without, _ = R.bwd(logits, ids, counts, tokens, tuple(0.0 if i == term else v for i, v in enumerate(dl)), None, **ref)
                assert np.any(np.abs(without - want) > 100 * (bal + z)), (dl, term)
    # with the scores: all three of a size
    dl = (0.5 * T, -0.25 * T)
    want, size = R.bwd(logits, ids, counts, tokens, dl, dw, **ref)
    l = logits.astype(np.float64)
    R_all = float(l.max() - l.min())
    bal, z = _bounds(logits, ids, counts, tokens, dl, off, mask, sigmoid)
    arrives = np.where((ids >= 0) & (ids < E), np.abs(dw), 0).sum(1)
    bound = bal + z + ((4 * R_all + 48) * U * arrives)[:, None]
    got = _run(logits, ids, dw, dl=dl, **opt)[4]
    assert np.all(np.abs(got - want) <= bound + 1e-30), np.abs(got - want).max()
    for term in (0, 1):
        if term or k < E:
            without, _ = R.bwd(logits, ids, counts, tokens, tuple(0.0 if i == term else v for i, v in enumerate(dl)), dw, **ref)
            assert np.any(np.abs(without - want) > bound), term


@pytest.mark.parametrize("T,E,k", SHAPES)
@pytest.mark.parametrize("sigmoid,renorm", [(False, True), (True, False)])
def test_one_sequence(T, E, k, sigmoid, renorm):
    logits, ids, dw = _case(T, E, k, T + 2 * E + k, dup=True)
    _check_terms(logits, ids, dw, sigmoid=sigmoid, renorm=renorm)


@pytest.mark.parametrize("sigmoid,renorm", [(False, False), (False, True), (True, True)])
@pytest.mark.parametrize("T,E,k,n", [(2000, 256, 8, 7), (700, 130, 6, 3), (515, 8, 2, 40), (64, 64, 6, 64), (1500, 48, 4, 1100), (900, 512, 4, 5)])
def test_sequences_and_masks(T, E, k, n, sigmoid, renorm):
    logits, ids, dw = _case(T, E, k, 7 * T + n, dup=True, bad=True)
    rng = np.random.default_rng(n)
    off = np.sort(rng.integers(T // 50, T - T // 40, size=n + 1)).astype(np.int32)
    mask = (rng.random(T) > 0.25).astype(np.uint8)
    mask[off[n // 2]:off[n // 2 + 1]] = 0
    _check_terms(logits, ids, dw, off, mask, sigmoid, renorm)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("T,E,k,n", [(40000, 64, 2, 1), (30000, 256, 4, 6), (9000, 1024, 8, 2), (65536, 8, 2, 3), (65536, 130, 1, 97)])
def test_means_and_losses_over_many_blocks(T, E, k, n, sigmoid):
    """A mean is a sum of a lane's rounds (up to 16), a warp's groups (5), a block's warps (32) and the blocks (148): 201 positive terms one
    after another at most, each sum off by half a unit."""
    from paper_2605_23764_b200 import MoeLayer
    rng = np.random.default_rng(T + E)
    logits = torch.from_numpy(rng.normal(size=(T, E)).astype(np.float32)).cuda()
    ids = torch.topk(logits, k, dim=1).indices.to(torch.int32).contiguous()
    off = [0] + sorted(int(v) for v in rng.integers(0, T, size=n - 1)) + [T]
    layer = MoeLayer(T, 64, E, k, 0, 64, sigmoid_gate=sigmoid)
    losses, counts, prob, tokens = layer.balance_fwd(logits, ids, torch.tensor(off, dtype=torch.int32).cuda() if n > 1 else None)
    layer.close()
    l = logits.double()
    p = torch.sigmoid(l) if sigmoid else torch.softmax(l, 1)
    p = p / p.sum(1, keepdim=True)
    spread, most = float((l.amax(1) - l.amin(1)).max()), float(l.abs().max())
    e = (2 * (spread + most) + 16) * U
    balance = 0.0
    for s, (a, b) in enumerate(zip(off[:-1], off[1:])):
        c = torch.bincount(ids[a:b].reshape(-1).long(), minlength=E)
        assert torch.equal(counts[s].long(), c) and int(tokens[s]) == b - a
        if b > a:
            mean = p[a:b].mean(0)
            assert float(((prob[s] - mean).abs() / mean).max()) <= e + 101 * U
            balance += E / (k * (b - a)) * float((c * mean).sum()) / n
    assert abs(float(losses[0]) - balance) <= (e + 108 * U) * balance
    # a squared logsumexp is off by twice its value times e + its own rounding; the sum as above
    lse = torch.logsumexp(l, 1)
    rms = float((lse ** 2).mean()) ** 0.5
    assert abs(float(losses[1]) - rms ** 2) <= 2 * rms * (e + float(lse.abs().max()) * U) + 108 * U * rms ** 2
