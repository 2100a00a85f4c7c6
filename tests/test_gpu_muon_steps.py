"""More steps and other polynomials through both kernels of the orthogonalised momentum, on spectra with singular values that are brought up
from far below the largest.

Tolerance.  Singular values far below the largest grow by the linear coefficient a step, and what roundings relative to the large ones add to them
grows with them.  X's second part is to be kept until the products of the |a| that are left, from every step's to the last's, sum up to at most 16: a rounding
to 11 bits has a root mean square of 2^-11 / sqrt(3) of the entry, and 16 of them are 4.5e-3 of the result's norm, which is not below
that of the large values.  On top of what the few first steps' tolerance covers (test_gpu_muon.py)."""
import pytest
import torch

from .test_gpu_muon import COEF, NORM, _exact, _near

pytestmark = pytest.mark.gpu
KEPT = 16 * 2.0 ** -11 / 3 ** 0.5
Q, C = (1.875, -1.25, 0.375), (1.5, -0.5, 0.0)


def _spectrum(rows, cols, kind):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    m = min(rows, cols)
    a, b = torch.randn(rows, m, device="cuda", generator=g), torch.randn(m, cols, device="cuda", generator=g)
    if kind == "low_rank":      # the other singular values are what bf16 makes of zero
        G = a[:, :m // 4] @ b[:m // 4]
    elif kind == "one_large":
        G = 40 * a[:, :1] @ b[:1] + 0.1 * torch.randn(rows, cols, device="cuda", generator=g)
    elif kind == "steep":
        G = (a * torch.logspace(0, -4, m, device="cuda")) @ b
    else:
        G = a @ b
    return G.to(torch.bfloat16)[None].contiguous()


@pytest.mark.parametrize("rows,cols", [(256, 400), (400, 256), (264, 1056), (120, 200), (48, 96)])
@pytest.mark.parametrize("kind", ["low_rank", "one_large", "steep", "full"])
@pytest.mark.parametrize("coef,steps", [(COEF, 6), (COEF, 7), (COEF, 9), (Q, 8), (Q, 12), (C, 12), (C, 16), ([COEF] * 5 + [Q] * 3, 8),
                                        ([(4.0, -7.0, 3.5), (3.5, -5.0, 2.2)] + [Q] * 4, 6)])
def test_small_singular_values_brought_up_by_many_steps(rows, cols, kind, coef, steps):
    from paper_2605_23764_b200 import MoeMuon
    G = _spectrum(rows, cols, kind)
    muon = MoeMuon(1, rows, cols, coefficients=coef, steps=steps)
    out = muon.orthogonalize(G)
    assert muon.status() == (0, 0)
    _near(out, _exact(G, coef, steps), NORM + KEPT)
