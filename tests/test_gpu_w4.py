"""The layer over 4-bit weights, and the weights' way into them, against numpy in 64 bits (tolerances: w4_ref.layer)."""
import numpy as np
import pytest
import torch

from . import w4_ref as R

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _cuda(a, dtype=None):
    return None if a is None else torch.as_tensor(np.ascontiguousarray(a), dtype=dtype).cuda()


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,rows,cols,gate_up", [(1, 16, 64, False), (3, 1, 8, False), (2, 40, 200, False), (2, 48, 136, True), (1, 7, 712, False),
                                                 (5, 16, 1160, True), (2, 130, 72, False)])
def test_packed_codes_come_back_as_their_values(n, rows, cols, gate_up, group, asym):
    from paper_2605_23764_b200 import MoeW4Weights
    rng = np.random.default_rng(n * rows + cols + group)
    q, s, z = R.random_codes(rng, n, rows, cols, group, asym)
    w = MoeW4Weights.pack(_cuda(q), _cuda(s, BF), _cuda(z), group=group, gate_up=gate_up)
    got = w.dequantize().float().cpu().numpy()
    assert np.array_equal(got, R.bf16(R.values(q, s, z, group).astype(np.float32)))   # the product is exact in fp32


@pytest.mark.parametrize("asym", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,rows,cols,gate_up", [(1, 16, 64, False), (2, 33, 8, False), (2, 64, 328, True), (3, 16, 712, False)])
def test_quantized_weights(n, rows, cols, gate_up, group, asym):
    from paper_2605_23764_b200 import MoeW4Weights
    rng = np.random.default_rng(rows + cols + group)
    W = R.bf16(rng.normal(size=(n, rows, cols)) * np.exp(rng.normal(size=(n, rows, 1))))
    W[0, 0] = 0                      # a group of zeros
    W[-1, -1] = np.abs(W[-1, -1])    # of one sign
    W[0, rows // 2, ::3] = -0.0
    w = MoeW4Weights.quantize(_cuda(W, BF), group=group, asymmetric=asym, gate_up=gate_up)
    got = w.dequantize().float().cpu().numpy()
    want = R.quantized(W, group, asym)
    assert np.array_equal(got, R.bf16(want.astype(np.float32)))
    # half a step of the group's scale at most, a rounded scale's share of the largest code, and the bf16 value's rounding
    step = np.abs(W).max() * (2.0 if asym else 1.0) / (15 if asym else 7)
    assert np.abs(got - W).max() <= step * (0.5 + 15 * 2.0 ** -8 + (0.5 if asym else 0.0)) + 2.0 ** -8 * np.abs(W).max()


def _problem(T, d, E, k, S, F, group, asym, seed, ids=None):
    rng = np.random.default_rng(seed)
    x = R.bf16(rng.normal(size=(T, d)))
    up, down = R.random_codes(rng, E + S, 2 * F, d, group, asym), R.random_codes(rng, E + S, d, F, group, asym)
    if ids is None:
        ids = np.argsort(rng.random((T, E)), 1)[:, :k].astype(np.int32).reshape(T, k)
    w = rng.random((T, k)).astype(np.float32)
    return x, ids, w, up, down


def _weights(up, down, group):
    from paper_2605_23764_b200 import MoeW4Weights
    pack = lambda p, gu: MoeW4Weights.pack(_cuda(p[0]), _cuda(p[1], BF), _cuda(p[2]), group=group, gate_up=gu)
    return pack(up, True), pack(down, False)


def _run(T, d, E, k, S, F, x, ids, w, up, down, group, T_max=None, status=(0, 0)):
    from paper_2605_23764_b200 import MoeLayer
    layer = MoeLayer(T_max or T, d, E, k, S, F, w4=True)
    W1, W2 = _weights(up, down, group)
    out = layer.ffn_fwd_w4(_cuda(x, BF), _cuda(ids), _cuda(w), W1, W2)
    torch.cuda.synchronize()
    got = layer.status()
    assert got == status or (status[1] is None and got[0] == status[0])
    layer.close()
    return out.float().cpu().numpy()


def _check(got, x, ids, w, up, down, group, E):
    # some experts' weights may be rounded to bf16 on the way: bounded as if all were
    want, bound = R.layer(x, ids, w, R.values(*up, group), R.values(*down, group), E, rounded_weights=True)
    assert np.isfinite(got).all()
    bad = np.abs(got - want) > bound
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5], np.abs(got - want).max(), np.abs(want).max())
    # five roundings to bf16 of independent signs, each 2^-8 / sqrt(3) of its value at most in the mean square
    norm = np.linalg.norm(want)
    assert np.linalg.norm(got - want) <= 2.0 ** -8 * (5 / 3) ** 0.5 * norm


SHAPES = [   # T, d, E, k, S, F
    (1, 64, 4, 1, 0, 32), (1, 8, 1, 1, 0, 8), (1, 256, 8, 2, 1, 128), (2, 72, 4, 4, 0, 24), (5, 200, 3, 2, 2, 40), (8, 512, 16, 4, 1, 200),
    (9, 128, 8, 8, 0, 64), (17, 136, 24, 3, 1, 72), (33, 256, 2, 1, 0, 128), (64, 328, 64, 6, 2, 136), (200, 192, 8, 2, 1, 64), (333, 104, 5, 3, 0, 88),
]


@pytest.mark.parametrize("asym,group", [(False, 128), (True, 64), (False, 32), (True, 32), (True, 128), (False, 64)])
@pytest.mark.parametrize("T,d,E,k,S,F", SHAPES)
def test_layer(T, d, E, k, S, F, group, asym):
    p = _problem(T, d, E, k, S, F, group, asym, T + d + E + F)
    _check(_run(T, d, E, k, S, F, *p, group), *p, group, E)


@pytest.mark.parametrize("T,d,E,k,S,F", [(1, 2048, 8, 6, 1, 1408), (4, 7168, 3, 2, 1, 520), (40, 2048, 6, 3, 1, 1408), (300, 1024, 10, 4, 1, 704)])
def test_long_rows(T, d, E, k, S, F):
    p = _problem(T, d, E, k, S, F, 128, False, T + d)
    _check(_run(T, d, E, k, S, F, *p, 128), *p, 128, E)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T", [10, 11, 20, 21, 40, 41])
def test_either_side_of_the_vector_kernels_slots(T, group):
    """Slots from 80 to 328: what the two kernels share of a batch does not depend on its length by more than their roundings."""
    d, E, k, S, F = 136, 90, 7, 1, 72
    p = _problem(T, d, E, k, S, F, group, True, 5)
    _check(_run(T, d, E, k, S, F, *p, group), *p, group, E)


@pytest.mark.parametrize("T", [1, 3, 40])
@pytest.mark.parametrize("groups", [(32, 128), (128, 32), (64, 32)])
def test_groups_of_their_own_for_either_product(groups, T):
    d, E, k, S, F = 200, 24, 2, 1, 136
    rng = np.random.default_rng(T)
    x, ids, w, up, _ = _problem(T, d, E, k, S, F, groups[0], False, T)
    down = R.random_codes(rng, E + S, d, F, groups[1], True)
    from paper_2605_23764_b200 import MoeLayer, MoeW4Weights
    W1 = MoeW4Weights.pack(_cuda(up[0]), _cuda(up[1], BF), None, group=groups[0], gate_up=True)
    W2 = MoeW4Weights.pack(_cuda(down[0]), _cuda(down[1], BF), _cuda(down[2]), group=groups[1])
    layer = MoeLayer(T, d, E, k, S, F, w4=True)
    got = layer.ffn_fwd_w4(_cuda(x, BF), _cuda(ids), _cuda(w), W1, W2).float().cpu().numpy()
    assert layer.status() == (0, 0)
    layer.close()
    want, bound = R.layer(x, ids, w, R.values(*up, groups[0]), R.values(*down, groups[1]), E, rounded_weights=True)
    assert (np.abs(got - want) <= bound).all()


@pytest.mark.parametrize("T,d,F,group", [(1, 40000, 8, 128), (1, 8, 40000, 32), (2, 26000, 16, 32), (5, 45056, 24, 64)])
def test_rows_longer_than_shared_memory(T, d, F, group):
    p = _problem(T, d, 3, 2, 1, F, group, True, T + d)
    _check(_run(T, d, 3, 2, 1, F, *p, group), *p, group, 3)


@pytest.mark.parametrize("rows", [7, 8, 9, 16, 31, 32, 33, 100, 128, 129, 192, 193, 257])
def test_one_expert_takes_all(rows):
    d, E, F = 136, 40, 72
    ids = np.full((rows, 1), 17, np.int32)
    p = _problem(rows, d, E, 1, 0, F, 64, True, rows, ids)
    _check(_run(rows, d, E, 1, 0, F, *p, 64), *p, 64, E)


def test_uneven_experts():
    """Experts without a row, with one, with a few and with hundreds in one call."""
    T, d, E, k, F = 700, 128, 12, 2, 72
    rng = np.random.default_rng(8)
    ids = np.stack([rng.choice(E, size=2, replace=False, p=np.array([400, 150, 60, 30, 10, 8, 4, 2, 1, 1, 0, 0]) / 666) for _ in range(T)]).astype(np.int32)
    p = _problem(T, d, E, k, 1, F, 128, False, 3, ids)
    _check(_run(T, d, E, k, 1, F, *p, 128), *p, 128, E)


@pytest.mark.parametrize("T", [3, 150])
def test_ids_named_twice_and_out_of_range(T):
    d, E, k, S, F = 96, 6, 3, 1, 40
    p = list(_problem(T, d, E, k, S, F, 32, True, 77))
    ids = p[1]
    ids[:, 1] = ids[:, 0]
    ids[1, 2] = -1
    ids[T - 1, 0] = E
    got = _run(T, d, E, k, S, F, *p, 32, status=(1, None))
    _check(got, *p, 32, E)


def test_a_shorter_batch_than_the_context_and_repeated_calls():
    from paper_2605_23764_b200 import MoeLayer
    d, E, k, S, F, group = 256, 16, 4, 1, 128, 64
    layer = MoeLayer(300, d, E, k, S, F, w4=True)
    base = _problem(1, d, E, k, S, F, group, False, 0)
    W1, W2 = _weights(base[3], base[4], group)
    for T in (300, 1, 64, 2, 257, 13, 300, 0):
        x, ids, w, _, _ = _problem(max(T, 1), d, E, k, S, F, group, False, T)
        x, ids, w = x[:T], ids[:T], w[:T]
        out = layer.ffn_fwd_w4(_cuda(x, BF), _cuda(ids), _cuda(w), W1, W2)
        again = layer.ffn_fwd_w4(_cuda(x, BF), _cuda(ids), _cuda(w), W1, W2)
        assert torch.equal(out, again) and layer.status() == (0, 0)
        if T:
            _check(out.float().cpu().numpy(), x, ids, w, base[3], base[4], group, E)
    layer.close()


def test_rows_behind_the_batch_stay():
    from paper_2605_23764_b200 import MoeLayer, binding as B
    T, d, E, k, F, group = 5, 64, 4, 2, 32, 32
    p = _problem(T, d, E, k, 0, F, group, False, 1)
    W1, W2 = _weights(p[3], p[4], group)
    layer = MoeLayer(16, d, E, k, 0, F, w4=True)
    out = torch.full((16, d), 7.0, dtype=BF).cuda()
    B.moe_ffn_fwd_w4(layer.ctx, _cuda(p[0], BF), _cuda(p[1]), _cuda(p[2]), W1, W2, out, T)
    assert bool((out[T:] == 7).all())
    _check(out[:T].float().cpu().numpy(), *p, group, E)
    layer.close()


@pytest.mark.parametrize("T", [4, 200])
def test_graphs_and_streams(T):
    from paper_2605_23764_b200 import MoeLayer
    d, E, k, S, F, group = 256, 8, 2, 1, 128, 128
    p = _problem(T, d, E, k, S, F, group, True, T)
    W1, W2 = _weights(p[3], p[4], group)
    layers = [MoeLayer(T, d, E, k, S, F, w4=True) for _ in range(2)]
    x, ids, w = _cuda(p[0], BF), _cuda(p[1]), _cuda(p[2])
    want = layers[0].ffn_fwd_w4(x, ids, w, W1, W2)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for s, layer in zip(streams, layers):   # two contexts at once
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs += [layer.ffn_fwd_w4(x, ids, w, W1, W2) for _ in range(5)]
    torch.cuda.synchronize()
    assert all(torch.equal(want, o) for o in outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layers[0].ffn_fwd_w4(x, ids, w, W1, W2)
    other = _problem(T, d, E, k, S, F, group, True, T + 1)
    for q in (p, other):
        x.copy_(_cuda(q[0], BF)); ids.copy_(_cuda(q[1])); w.copy_(_cuda(q[2]))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        _check(out.float().cpu().numpy(), q[0], q[1], q[2], p[3], p[4], group, E)
    for layer in layers:
        assert layer.status() == (0, 0)
        layer.close()


def test_serving_route_and_4_bit_layer_next_to_the_bf16_layer():
    """Weights quantized once, routing and layer step by step; the bf16 layer over the same values agrees, and its saved forward is given up."""
    from paper_2605_23764_b200 import MoeError, MoeLayer, MoeW4Weights
    T, d, E, k, S, F = 96, 256, 16, 4, 1, 128
    g = torch.Generator().manual_seed(3)
    W1 = (torch.randn(E + S, 2 * F, d, generator=g) / d ** 0.5).to(BF).cuda()
    W2 = (torch.randn(E + S, d, F, generator=g) / F ** 0.5).to(BF).cuda()
    q1, q2 = MoeW4Weights.quantize(W1, group=64, gate_up=True), MoeW4Weights.quantize(W2, group=64, asymmetric=True)
    layer = MoeLayer(T, d, E, k, S, F, renorm=True, save_for_bwd=True, w4=True)
    v1, v2 = q1.dequantize(), q2.dequantize()
    for n in (T, 1, 9):
        x = torch.randn(n, d, generator=g).to(BF).cuda()
        ids, w = layer.route(torch.randn(n, E, generator=g).cuda())
        want = layer.ffn_fwd(x, ids, w, v1, v2).float()
        got = layer.ffn_fwd_w4(x, ids, w, q1, q2).float()
        # both round activations and rows, the bf16 layer its weights too: six roundings of 2^-8 / sqrt(3)
        assert float((got - want).norm()) <= 2.0 ** -8 * 2 ** 0.5 * float(want.norm())
        with pytest.raises(MoeError):
            layer.ffn_bwd(x, x, ids, w, v1, v2)
    # and the weights themselves: 4 bits of a normal law in groups of 64 keep about 0.12 of its deviation as error
    assert float((v1.float() - W1.float()).norm() / W1.float().norm()) < 0.2
    assert layer.status() == (0, 0)
    layer.close()


def test_refusals():
    from paper_2605_23764_b200 import MoeError, MoeLayer, MoeW4Weights
    T, d, E, k, F = 4, 64, 4, 2, 32
    p = _problem(T, d, E, k, 0, F, 32, False, 1)
    W1, W2 = _weights(p[3], p[4], 32)
    x, ids, w = _cuda(p[0], BF), _cuda(p[1]), _cuda(p[2])
    plain = MoeLayer(T, d, E, k, 0, F)
    with pytest.raises(MoeError):                      # no room in the workspace
        plain.ffn_fwd_w4(x, ids, w, W1, W2)
    plain.close()
    layer = MoeLayer(T, d, E, k, 0, F, w4=True)
    with pytest.raises(MoeError, match="W_down"):
        layer.ffn_fwd_w4(x, ids, w, W1, W1)
    with pytest.raises(MoeError, match="W_gate_up"):
        layer.ffn_fwd_w4(x, ids, w, torch.zeros(1).cuda(), W2)
    with pytest.raises(MoeError, match="topk_ids"):
        layer.ffn_fwd_w4(x, ids.long(), w, W1, W2)
    with pytest.raises(MoeError):
        layer.ffn_fwd_w4(x.repeat(2, 1), ids.repeat(2, 1), w.repeat(2, 1), W1, W2)   # more than T_max
    odd = torch.empty(T * d + 1, dtype=BF, device="cuda")[1:].view(T, d)
    with pytest.raises(MoeError):                      # not 16-byte aligned
        layer.ffn_fwd_w4(odd, ids, w, W1, W2)
    with pytest.raises(MoeError, match="contiguous"):
        MoeW4Weights.quantize(torch.zeros(1, 64, 32, dtype=BF).cuda().transpose(1, 2))
    with pytest.raises(MoeError):
        MoeW4Weights.quantize(torch.zeros(1, 16, 64, dtype=BF).cuda(), group=100)
    layer.close()
