"""The layer over 4-bit weights with as many experts as a context may have."""
import pytest

from .test_gpu_w4 import _check, _problem, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 3, 4, 40])   # three tokens are 288 slots, four 384: one kernel, the other
@pytest.mark.parametrize("asym,group", [(False, 32), (True, 128)])
def test_most_experts(T, asym, group):
    d, E, k, S, F = 64, 1024, 32, 64, 32
    p = _problem(T, d, E, k, S, F, group, asym, T)
    _check(_run(T, d, E, k, S, F, *p, group), *p, group, E)
