"""Weights at the two ends of bf16's range: quantizing does not depend on a power of two."""
import numpy as np
import pytest
import torch

from . import w4_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("asym", [False, True])
def test_weights_whose_range_is_beyond_fp32(asym, group):
    """Finite weights from -1.6e38 to 3.2e38: the range of a group is 4.8e38, its scale 3.2e37."""
    from paper_2605_23764_b200 import MoeW4Weights
    rng = np.random.default_rng(group)
    W = R.bf16(rng.random((2, 48, 264)) * 4.8e38 - 1.6e38)
    W[:, ::2, ::group] = R.bf16(np.float32(-1.6e38))
    W[:, ::2, group - 1::group] = R.bf16(np.float32(3.2e38))
    assert np.isfinite(W).all()
    got = MoeW4Weights.quantize(torch.from_numpy(W).to(torch.bfloat16).cuda(), group=group, asymmetric=asym).dequantize().float().cpu().numpy()
    want = R.quantized(W * np.float32(2.0 ** -40), group, asym) * 2.0 ** 40
    assert np.isfinite(got).all()
    assert np.array_equal(got, R.bf16(want.astype(np.float32)))


@pytest.mark.parametrize("asym", [False, True])
def test_weights_near_the_smallest(asym):
    """Scales down to the smallest normal number of bf16, and below it."""
    from paper_2605_23764_b200 import MoeW4Weights
    rng = np.random.default_rng(4)
    W = R.bf16(rng.normal(size=(1, 64, 128)) * 2.0 ** -rng.integers(90, 130, size=(1, 64, 1)))
    got = MoeW4Weights.quantize(torch.from_numpy(W).to(torch.bfloat16).cuda(), group=64, asymmetric=asym).dequantize().float().cpu().numpy()
    assert np.array_equal(got, R.bf16(R.quantized(W, 64, asym).astype(np.float32)))
