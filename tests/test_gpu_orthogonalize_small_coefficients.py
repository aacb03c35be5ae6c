"""Orthogonalised updates with steps whose polynomial is all but linear: coefficients far below the words' exponents, down to
FP32's smallest.  What they add is below every rounding, so the result is that of the other coefficients.

Bounds: those of the polynomial in 64 bits, with the same allowance for every step."""
import pytest
import torch

from test_gpu_orthogonalize import DEV, bound, check, h, rand, steps_of  # noqa: F401  (h: the handle's fixture)

pytestmark = pytest.mark.gpu

CUBIC = (1.5, -0.5, 0.0)
STEPS = [[(1.0, 1e-36, 0.0)], [(1.5, 1e-35, 0.0)], [(2.0, 0.0, -3e-38)], [(1.0, 1e-45, 1e-45)], [(0.75, -1e-20, 1e-20)], [(1.0, 0.0, 0.0)],
         [CUBIC, (1.0, 1e-36, 0.0), CUBIC], [(1024.0, 0.0, 0.0), (2.0 ** -10, 1e-41, 0.0), CUBIC]]


# one launch; a launch for every product, wide and tall
@pytest.mark.parametrize("rows,cols", [(1, 1), (90, 140), (140, 90), (300, 1000), (2301, 2500), (2500, 2301)])
@pytest.mark.parametrize("coefficients", STEPS)
def test_steps_that_are_all_but_linear(h, rows, cols, coefficients):  # noqa: F811
    g = rand(31, rows, cols)
    got = check(h, g, len(coefficients), coefficients=coefficients)
    # (the smallest coefficients left out: the same matrix but for the roundings of one result)
    linear = [(a, b if abs(b) > 1e-30 else 0.0, c if abs(c) > 1e-30 else 0.0) for a, b, c in coefficients]
    want = steps_of(g, torch.float64, len(coefficients), linear)
    assert bool(torch.isfinite(got).all())
    assert float((got.double() - want).norm()) <= bound(rows, cols, len(coefficients)) * float(want.norm())


def test_steps_of_the_largest_and_smallest_singular_values(h):  # noqa: F811
    """Singular values of 2^20 and of 2^-20 at the largest, the ends of what a step may leave, and back."""
    for up in (2.0 ** 19.5, 2.0 ** -19.5):
        for coefficients in ([(up, 0.0, 0.0), (1.0 / up, 0.0, 0.0)], [(up, 0.0, 0.0), (0.0, up ** -3, 0.0)],
                             [(up, 0.0, 0.0), (1.0 / up, 1e-45, 0.0), CUBIC]):
            # X = G X0 with one direction only: the polynomial of one number, every entry of the result at its own size
            g = torch.zeros(40, 70, device=DEV)
            g[3, 7], g[3, 8] = 3.0, 4.0
            got = torch.full_like(g, float("nan"))
            h.sgemm_cube_orthogonalize(g, got, steps=len(coefficients), coefficients=coefficients)
            want = steps_of(g, torch.float64, len(coefficients), coefficients)
            assert float((got.double() - want).norm()) <= bound(40, 70, len(coefficients)) * float(want.norm()), (up, coefficients)
