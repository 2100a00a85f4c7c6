"""4-bit weights: sizes and refusals, without a GPU."""
import pytest
import torch

from paper_2605_23764_b200 import MoeError, binding as B, build


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def test_sizes():
    assert B.moe_w4_sizes(128, 128, 64) == (8192, 256)
    assert B.moe_w4_sizes(16, 64, 32) == (8192, 512)
    assert B.moe_w4_sizes(129, 136, 128) == (4 * 8192, 4 * 128)      # rows to 128, columns to 128
    assert B.moe_w4_sizes(4096, 7168, 128, B.MOE_W4_GATE_UP) == (4096 * 7168 // 2, 4096 * 56)
    for bad in ((0, 64, 64, 0), (16, 0, 64, 0), (16, 60, 64, 0), (16, 64, 16, 0), (16, 64, 256, 0), (24, 64, 64, 1), (16, 64, 64, 2)):
        with pytest.raises(MoeError):
            B.moe_w4_sizes(*bad)


def test_the_flag_makes_room():
    plain = B.moe_workspace_bytes(64, 256, 8, 2, 1, 128)
    assert B.moe_workspace_bytes(64, 256, 8, 2, 1, 128, B.MOE_FLAG_W4) >= plain + 64 * 3 * 256 * 4


def test_binding_refuses_what_does_not_fit():
    bf, u8 = torch.bfloat16, torch.uint8
    nb, ne = B.moe_w4_sizes(32, 64, 32)
    codes, scales, zeros = torch.zeros(2, nb // 4, dtype=torch.int32), torch.zeros(2, ne, dtype=bf), torch.zeros(2, ne, dtype=u8)
    W = torch.zeros(2, 32, 64, dtype=bf)
    with pytest.raises(MoeError, match="codes"):
        B.moe_w4_quantize(W, 2, 32, 64, 32, 0, codes[:1], scales, None)
    with pytest.raises(MoeError, match="scales"):
        B.moe_w4_quantize(W, 2, 32, 64, 32, 0, codes, scales[:1], None)
    with pytest.raises(MoeError, match="zeros"):
        B.moe_w4_quantize(W, 2, 32, 64, 32, 0, codes, scales, zeros[:1])
    with pytest.raises(MoeError, match="W:"):
        B.moe_w4_quantize(W[:1], 2, 32, 64, 32, 0, codes, scales, zeros)
    with pytest.raises(MoeError, match="CUDA"):                     # sizes fit: no CPU tensor reaches a kernel
        B.moe_w4_quantize(W, 2, 32, 64, 32, 0, codes, scales, zeros)
    q, qs = torch.zeros(2, 32, 32, dtype=u8), torch.zeros(2, 32, 2, dtype=bf)
    with pytest.raises(MoeError, match="q_scales"):
        B.moe_w4_pack(q, qs[:, :, :1].contiguous(), None, 2, 32, 64, 32, 0, codes, scales, None)
    with pytest.raises(MoeError, match="q_zeros"):
        B.moe_w4_pack(q, qs, torch.zeros(2, 32, 1, dtype=u8), 2, 32, 64, 32, 0, codes, scales, zeros)
    with pytest.raises(MoeError, match="W:"):
        B.moe_w4_dequantize(codes, scales, zeros, 32, 2, 32, 64, 0, W[:1])
    with pytest.raises(MoeError, match="n matrices"):
        B.MoeW4Weights.quantize(W[0])
    with pytest.raises(MoeError):
        B.MoeW4Weights.quantize(torch.zeros(1, 24, 64, dtype=bf), gate_up=True)   # 12 features


def test_entry_points_refuse_before_they_launch():
    """Straight at the C entry points, on the host."""
    import ctypes
    lib = B.load_library()
    INVALID = -1
    p = lambda v: ctypes.c_void_p(v)
    assert lib.moe_w4_quantize(p(256), 1, 16, 64, 48, 0, p(256), p(256), None, None) == INVALID
    assert lib.moe_w4_quantize(p(264), 1, 16, 64, 64, 0, p(256), p(256), None, None) == INVALID   # not 16-byte aligned
    assert lib.moe_w4_quantize(p(256), 1, 16, 64, 64, 0, p(256), None, None, None) == INVALID
    assert lib.moe_w4_quantize(p(256), -1, 16, 64, 64, 0, p(256), p(256), None, None) == INVALID
    assert lib.moe_w4_quantize(None, 0, 16, 64, 64, 0, None, None, None, None) == 0
    assert lib.moe_w4_pack(p(256), p(256), None, 1, 16, 64, 64, 0, p(256), p(256), p(256), None) == INVALID   # zero points on one side
    assert lib.moe_w4_pack(p(257), p(256), None, 1, 16, 64, 64, 0, p(256), p(256), None, None) == INVALID
    w = B._W4(256, 256, None, 40)
    assert lib.moe_w4_dequantize(ctypes.byref(w), 1, 16, 64, 0, p(256), None) == INVALID
    assert lib.moe_ffn_fwd_w4(None, None, None, None, None, None, None, 1, None) == INVALID
    assert lib.moe_balance_fwd(None, p(256), p(256), 1, None, 1, None, p(256), p(256), p(256), p(256), None) == INVALID
    assert lib.moe_balance_bwd(None, p(256), p(256), p(256), p(256), p(256), None, 1, None, 1, None, p(256), None) == INVALID


def test_layer_calls_check_sizes_against_the_context():
    import ctypes
    fake = ctypes.c_void_p(54321)
    T, d, E, k, S, F = 8, 64, 4, 2, 1, 32
    B._CTX_SHAPE[fake.value] = (T, d, E, k, S, F, B.MOE_FLAG_W4)
    try:
        bf = torch.bfloat16
        up, down = B.MoeW4Weights(E + S, 2 * F, d, 64, True, False, "cpu"), B.MoeW4Weights(E + S, d, F, 32, False, True, "cpu")
        x, ids, w, out = torch.zeros(T, d, dtype=bf), torch.zeros(T, k, dtype=torch.int32), torch.zeros(T, k), torch.zeros(T, d, dtype=bf)
        with pytest.raises(MoeError, match="W_down"):
            B.moe_ffn_fwd_w4(fake, x, ids, w, up, up, out, T)
        with pytest.raises(MoeError, match="W_gate_up"):
            B.moe_ffn_fwd_w4(fake, x, ids, w, B.MoeW4Weights(E + S, 2 * F, d, 64, False, False, "cpu"), down, out, T)
        with pytest.raises(MoeError, match="out"):
            B.moe_ffn_fwd_w4(fake, x, ids, w, up, down, out[:-1], T)
        down.zeros = down.zeros[:, :-1]
        with pytest.raises(MoeError, match="zeros"):
            B.moe_ffn_fwd_w4(fake, x, ids, w, up, down, out, T)
        with pytest.raises(MoeError, match="tokens"):
            B.moe_balance_fwd(fake, torch.zeros(T, E), ids, T, torch.zeros(3, dtype=torch.int32), 2, None, torch.zeros(2),
                              torch.zeros(2, E, dtype=torch.int32), torch.zeros(2, E), torch.zeros(2, dtype=torch.int32))
    finally:
        B._CTX_SHAPE.pop(fake.value)
