"""Sizes beyond 32 bits, or so near to them that rounding up would leave them, are refused and not cut off."""
import ctypes

import pytest
import torch

from paper_2605_23764_b200 import MoeError, binding as B, build


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def test_sizes_at_the_limits():
    most = 2**31 - 1 - 128
    big = most // 16 * 16
    for flags in (0, B.MOE_W4_GATE_UP):
        for rows, cols in ((big, 8), (16, big), (big, big)):
            tiles, units = -(-rows // 128) * 4, -(-cols // 128)
            assert B.moe_w4_sizes(rows, cols, 32, flags) == (tiles * units * 2048, tiles * units * 4 * 32)
    assert B.moe_w4_sizes(most, 64, 128)[1] == -(-most // 128) * 128
    for rows, cols in ((most + 1, 64), (2**31 - 1, 64), (16, 2**31 - 8), (2**32 + 16, 64), (16, 2**32 + 64), (2**64 + 16, 64)):
        with pytest.raises(MoeError):
            B.moe_w4_sizes(rows, cols, 64)


def test_numbers_that_are_no_32_bit_numbers():
    """Ones that 32 bits would cut to a small number."""
    bf, i32, u8 = torch.bfloat16, torch.int32, torch.uint8
    many = 2**32 + 4
    wide = lambda t, *shape: t.expand(*shape)   # as many elements as needed, one in memory
    fake = ctypes.c_void_p(76543)
    d, E, k, F = 8, 1, 1, 8
    B._CTX_SHAPE[fake.value] = (8, d, E, k, 0, F, B.MOE_FLAG_W4)
    try:
        up, down = B.MoeW4Weights(1, 2 * F, d, 32, True, False, "cpu"), B.MoeW4Weights(1, d, F, 32, False, False, "cpu")
        ids, f32 = torch.zeros(1, 1, dtype=i32), torch.zeros(1, 1)
        with pytest.raises(MoeError, match="T: "):
            B.moe_ffn_fwd_w4(fake, wide(torch.zeros(1, 1, dtype=bf), many, d), wide(ids, many, k), wide(f32, many, k), up, down,
                             wide(torch.zeros(1, 1, dtype=bf), many, d), many)
        args = (wide(ids, many, k), many, None, 1, None, torch.zeros(2), torch.zeros(1, E, dtype=i32), torch.zeros(1, E), torch.zeros(2, dtype=i32))
        with pytest.raises(MoeError, match="T: "):
            B.moe_balance_fwd(fake, wide(f32, many, E), *args)
        with pytest.raises(MoeError, match="n_seq: "):
            B.moe_balance_fwd(fake, f32, ids, 1, wide(torch.zeros(1, dtype=i32), many + 1), many, None, torch.zeros(2), wide(ids, many, E), wide(f32, many, E),
                              wide(torch.zeros(1, dtype=i32), many + 1))
        with pytest.raises(MoeError, match="T: "):
            B.moe_balance_bwd(fake, wide(f32, many, E), None, torch.zeros(1, E, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(2), None, many, None, 1,
                              None, wide(f32, many, E))
    finally:
        B._CTX_SHAPE.pop(fake.value)
    nb, ne = B.moe_w4_sizes(16, 8, 32)
    codes, scales = wide(torch.zeros(1, 1, dtype=i32), many, nb // 4), wide(torch.zeros(1, 1, dtype=bf), many, ne)
    W = wide(torch.zeros(1, 1, 1, dtype=bf), many, 16, 8)
    with pytest.raises(MoeError, match="n: "):
        B.moe_w4_quantize(W, many, 16, 8, 32, 0, codes, scales, None)
    with pytest.raises(MoeError, match="n: "):
        B.moe_w4_dequantize(codes, scales, None, 32, many, 16, 8, 0, W)
    with pytest.raises(MoeError, match="n: "):
        B.moe_w4_pack(wide(torch.zeros(1, 1, 1, dtype=u8), many, 16, 4), wide(torch.zeros(1, 1, 1, dtype=bf), many, 16, 1), None, many, 16, 8, 32, 0, codes,
                      scales, None)


def test_the_workspace_has_room_for_the_rows_that_there_can_be():
    """One token of a layer of 257 experts hits nine of them."""
    def room(T, d, E, k, S, F):
        return B.moe_workspace_bytes(T, d, E, k, S, F, B.MOE_FLAG_W4) - B.moe_workspace_bytes(T, d, E, k, S, F)

    for T, d, E, k, S, F in ((1, 7168, 256, 8, 1, 2048), (8, 7168, 256, 8, 1, 2048), (64, 2048, 64, 6, 2, 1408), (4096, 2048, 64, 6, 2, 1408), (0, 64, 4, 2, 0, 32)):
        slots = T * (k + S)
        need = (slots + 127 * min(slots, E + S)) * d * 4
        assert need <= room(T, d, E, k, S, F) <= need + 512, (T, E)
