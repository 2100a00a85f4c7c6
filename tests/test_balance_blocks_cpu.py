"""How the forward of the balance losses is split, on the host."""
import pytest

from paper_2605_23764_b200 import binding as B, build


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def _round(E):
    """Tokens that a block takes at once: each warp one for every group of lanes that holds a row of 8, 16 or 32 values a lane."""
    if E <= 8:
        return 32 * 32
    lanes = 2
    while lanes < 32 and 16 * lanes < E:
        lanes *= 2
    warps = 24 if E <= 512 else 16
    while 5 * 4 * warps * E > 200 * 1024:   # counts and sums of every warp in shared memory
        warps //= 2
    return warps * (32 // lanes)


@pytest.mark.parametrize("E", [1, 7, 8, 9, 12, 16, 17, 32, 33, 64, 65, 100, 128, 129, 256, 257, 321, 500, 512, 513, 700, 1024])
def test_few_tokens_are_a_round_for_every_warp(E):
    n = _round(E)
    for T, blocks in ((0, 1), (1, 1), (n, 1), (n + 1, 2), (4 * n, 4), (100 * n - 1, 100), (148 * n, 148)):
        assert B.moe_debug_balance_blocks(T, E) == blocks, (E, T)
    for T in (148 * n + 1, 1000 * n):   # more tokens are shared evenly between one block an SM
        each = -(-T // 148)
        assert B.moe_debug_balance_blocks(T, E) == -(-T // each), (E, T)
