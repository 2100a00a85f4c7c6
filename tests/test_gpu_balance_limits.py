"""The balance losses at the ends of their sizes."""
import ctypes

import pytest
import torch

from .test_gpu_balance import _case, _check, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sigmoid,renorm", [(False, True), (True, False)])
@pytest.mark.parametrize("T,E,k", [(5, 1, 1), (2000, 1, 1), (33, 2, 2), (100, 3, 1), (1030, 7, 7), (40, 9, 9), (500, 1024, 32), (17, 32, 32)])
def test_fewest_and_most_experts(T, E, k, sigmoid, renorm):
    logits, ids, dw = _case(T, E, k, T + E)
    opt = dict(sigmoid=sigmoid, renorm=renorm)
    _check(_run(logits, ids, dw, **opt), logits, ids, dw, **opt)


def test_more_sequences_than_32_bits_can_step_over():
    """Straight at the C entry points: refused before anything is looked at, and the next call is a whole one."""
    from paper_2605_23764_b200 import MoeLayer, binding as B
    T, E, k = 16, 8, 2
    logits, ids, dw = _case(T, E, k, 1)
    layer = MoeLayer(T, 64, E, k, 0, 64)
    p, lib = ctypes.c_void_p(256), B.load_library()
    for n in (2**31 - 1, 2**30 + 1, 0, -1):
        for tokens in (T, 0):
            assert lib.moe_balance_fwd(layer.ctx, p, p, tokens, p, n, None, p, p, p, p, None) == -1
            assert lib.moe_balance_bwd(layer.ctx, p, p, p, p, p, None, tokens, p, n, None, p, None) == -1
    _check(_run(logits, ids, dw, layer=layer), logits, ids, dw)
    layer.close()
