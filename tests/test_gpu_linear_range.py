"""The few-row kernels of the linear layer at the ends of the FP32 range, against the definition in FP64.

The weight's scaling exponent must not show: a product or a partial sum may leave FP32 only where the
result's own terms do, and a finite result has to come out finite even then.  Tolerances (u = 2^-24): a sum
of K products in FP32 is off by at most max(2K, K + 14) u times the sum of the magnitudes (the latter for the
two-word representation of short sums), a sum that was taken again in FP64 by its words' 2^-22 of that."""
import math

import pytest
import torch

from paper_2507_23387_b200 import binding
from paper_2507_23387_b200.binding import WEIGHT_KN, WEIGHT_NK, PackedMatrix

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DEV = "cuda:0"
FORMS = [("packed", WEIGHT_NK), ("fp32", WEIGHT_NK), ("fp32", WEIGHT_KN)]


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    torch.cuda.synchronize()
    assert handle.sgemm_cube_check()[0] == 0
    handle.destroy()


def rand(seed, *shape, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV) * scale


def layer(h, x, w, form):
    """x w' (w: outputs x inputs) in the given form of the weight."""
    kind, layout = form
    w = w if layout == WEIGHT_NK else w.t().contiguous()
    if kind == "packed":
        p = PackedMatrix(*w.shape)
        h.sgemm_cube_pack(w, p)
        w = p
    n = w.shape[0] if layout == WEIGHT_NK else w.shape[1]
    y = torch.full((x.shape[0], n), float("nan"), device=DEV)
    h.sgemm_cube_linear(x, w, y, weight_layout=layout)
    return y


def product64(x, w):
    return x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()


@pytest.mark.parametrize("sx,sw", [(1e34, 1e-10), (1e34, 1e-25), (1e35, 1e-30), (1e37, 1e-37), (1e-30, 1e20), (1e30, 1e-25),
                                   (1e18, 1e18), (1e-20, 1e-15), (1e-12, 1e-12)])
@pytest.mark.parametrize("m", [1, 2, 3, 4])
@pytest.mark.parametrize("k", [192, 1001])
@pytest.mark.parametrize("form", FORMS)
def test_magnitudes(h, m, k, sx, sw, form):
    n = 70
    x, w = rand(1, m, k, scale=sx), rand(2, n, k, scale=sw)
    y = layer(h, x, w, form)
    want, mag = product64(x, w)
    assert torch.isfinite(y).all()
    assert bool(((y.double() - want).abs() <= max(2 * k, k + 14) * U * mag).all())


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("m", [1, 4])
def test_partial_sums_that_leave_the_range(h, m, form):
    """Terms of 2e38 of both signs, in an order in which FP32 sums meet infinity; the results are finite."""
    n, k = 33, 512
    x = torch.full((m, k), 2e38, device=DEV)
    x[:, k // 2:] *= -1.0                                     # first all positive, then all negative
    x += rand(3, m, k, scale=1e36)
    w = torch.ones(n, k, device=DEV)
    w[1::2] = -1.0
    y = layer(h, x, w, form)
    want, mag = product64(x, w)
    assert want.abs().max() < 3e38
    assert torch.isfinite(y).all()
    assert bool(((y.double() - want).abs() <= 2.0 ** -22 * mag + U * want.abs()).all())


@pytest.mark.parametrize("form", FORMS)
def test_products_that_leave_the_range(h, form):
    """Two products of 1e40 that take each other away."""
    n, k = 5, 300
    x, w = rand(4, 1, k), torch.ones(n, k, device=DEV)
    x[0, 7], x[0, 200] = 1e25, -1e25
    w[:, 7] = w[:, 200] = 1e15
    y = layer(h, x, w, form)
    want, mag = product64(x, w)
    assert torch.isfinite(y).all()
    assert bool(((y.double() - want).abs() <= 2.0 ** -22 * mag + U * want.abs()).all())


@pytest.mark.parametrize("form", FORMS)
def test_results_that_leave_the_range_and_nonfinite_entries(h, form):
    n, k = 40, 96
    x, w = rand(5, 4, k).abs() + 0.5, rand(6, n, k).abs() + 0.5
    x[0] *= 1e20
    w[3] *= 1e20                                              # one output of the first row above FP32
    x[1, 5], x[2, 0] = math.inf, math.nan
    x[3] = 0.0
    y = layer(h, x, w, form)
    assert y[0, 3] == math.inf and torch.isfinite(y[0, :3]).all() and torch.isfinite(y[0, 4:]).all()
    assert not torch.isfinite(y[1]).any() and torch.isnan(y[2]).all()
    assert bool((y[3] == 0).all())
