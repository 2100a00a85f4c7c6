"""Sizes and refusals of the orthogonalised momentum that need no GPU."""
import pytest
import torch

from paper_2605_23764_b200 import binding, build

COEF = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def test_workspace():
    size = lambda *a, **o: binding.moe_muon_workspace_bytes(binding.moe_muon_shape(*a, o.get("c", COEF), o.get("steps", 5), o.get("eps", 1e-7)))
    one = size(1, 256, 512)
    assert one >= 4 * 2 * 256 * 512 + 2 * 2 * 256 * 256   # X twice in two parts, A and B
    assert size(8, 256, 512) > 4 * one
    assert size(1, 512, 256) == one
    assert size(1000, 2048, 7168) < 1.1 * 2 ** 30          # a batch at a time
    assert size(1, 65536, 65536) > 2 ** 34                  # sizes beyond 32 bits
    assert size(1, 3, 5) > 0
    for n, rows, cols in ((0, 8, 8), (-1, 8, 8), (1, 0, 8), (1, 8, -8), (1, 65537, 8), (1, 8, 65537), (65537, 8, 8)):
        assert size(n, rows, cols) == 0
    assert size(1, 8, 8, eps=-1e-9) == size(1, 8, 8, eps=float("nan")) == size(1, 8, 8, eps=float("inf")) == 0
    assert size(1, 8, 8, c=(1.0, float("nan"), 0.0)) == 0
    with pytest.raises(binding.MoeError, match="steps"):
        size(1, 8, 8, steps=17)
    with pytest.raises(binding.MoeError, match="steps"):
        size(1, 8, 8, steps=0)
    with pytest.raises(binding.MoeError, match="coefficients"):
        size(1, 8, 8, c=[(1.0, 0.0, 0.0)] * 4)
    with pytest.raises(binding.MoeError, match="32-bit"):
        size(2 ** 32 + 1, 8, 8)


def test_handles_and_tensors_are_looked_at_before_the_call():
    import ctypes
    fake = ctypes.c_void_p(4711)
    t = torch.zeros(2, 8, 8, dtype=torch.bfloat16)
    with pytest.raises(binding.MoeError, match="unknown muon"):
        binding.moe_muon_orthogonalize(fake, t, t)
    binding._MUON_ELEMS[fake.value] = 3 * 64
    try:
        with pytest.raises(binding.MoeError, match="G: 128 elements"):
            binding.moe_muon_orthogonalize(fake, t, t)
        with pytest.raises(binding.MoeError, match="W_out"):
            f = torch.zeros(3, 8, 8)
            b = f.to(torch.bfloat16)
            binding.moe_muon_step(fake, b, f, b, 0.9, True, 0.1, 0.0, 1.0, t, f)
    finally:
        binding._MUON_ELEMS.pop(fake.value)


def test_routing_by_groups_looks_at_sizes_first():
    import ctypes
    fake = ctypes.c_void_p(4712)
    binding._CTX_SHAPE[fake.value] = (16, 64, 8, 2, 0, 32, 0)
    try:
        g = binding.moe_route_groups(2, 1, 2, 1.0)
        ids, w = torch.zeros(16, 2, dtype=torch.int32), torch.zeros(16, 2)
        with pytest.raises(binding.MoeError, match="logits: 120"):
            binding.moe_route_grouped(fake, torch.zeros(15, 8), None, 16, g, ids, w)
        with pytest.raises(binding.MoeError, match="bias"):
            binding.moe_route_grouped(fake, torch.zeros(16, 8), torch.zeros(7), 16, g, ids, w)
        with pytest.raises(binding.MoeError, match="d_logits"):
            binding.moe_route_grouped_bwd(fake, torch.zeros(16, 8), ids, w, 16, 1.0, False, torch.zeros(16, 7))
        with pytest.raises(binding.MoeError, match="counts"):
            binding.moe_bias_update(fake, torch.zeros(8), torch.zeros(2, 7, dtype=torch.int32), 2, 1e-3, torch.zeros(8))
        with pytest.raises(binding.MoeError, match="32-bit"):
            binding.moe_route_groups(2 ** 33 + 1)
    finally:
        binding._CTX_SHAPE.pop(fake.value)
