"""How the coefficients of an orthogonalisation may be given."""
import numpy as np
import pytest
import torch

from paper_2605_23764_b200 import binding

COEF = (3.4445, -4.7750, 2.0315)


def _of(coefficients, steps=5):
    s = binding.moe_muon_shape(1, 8, 8, coefficients, steps, 1e-7)
    return [list(s.coefficients[i]) for i in range(steps)]


@pytest.mark.parametrize("given", [np.array(COEF), np.array(COEF, np.float32), [np.float32(v) for v in COEF], [np.float64(v) for v in COEF],
                                   torch.tensor(COEF).tolist(), np.array([COEF] * 5, np.float32), [np.array(COEF, np.float32)] * 5, torch.tensor([COEF] * 5)])
def test_numbers_of_other_kinds(given):
    assert _of(given) == _of(COEF)
    assert _of([2, 0, 0], 3) == [[2.0, 0.0, 0.0]] * 3


@pytest.mark.parametrize("given", [COEF[:2], [COEF[:2]] * 5, [COEF] * 4 + [1.0], 3.0, None, "abc", [("a", "b", "c")] * 5, [COEF] * 6])
def test_refusals(given):
    with pytest.raises(binding.MoeError, match="coefficients"):
        _of(given)
