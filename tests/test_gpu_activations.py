"""Activations and their slopes against FP64, in both tails, by themselves: z is what the layer itself stored, and the
slope is the bias gradient of a single row with dY = 1.

Tolerances (u = 2^-24), relative to the value where it is a product and not a difference.  Sigmoid forms: an exponential
of argument A (|z|, or 1.6 (|z| + 0.045 |z|^3)) is off by 3 A u from the roundings of its argument and 4 u of its own,
the reciprocal and three products by 6 u.  GELU: Phi's lower tail has A = z^2 / 2 with five roundings, 5 A u, and its
polynomial 24 u.  Slopes are sums of two such terms: the same, of the terms' sizes."""
import math

import pytest
import torch

from paper_2507_23387_b200 import binding
from paper_2507_23387_b200.binding import ACT_GELU, ACT_GELU_TANH, ACT_SILU, WEIGHT_KN

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DEV = "cuda:0"


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    torch.cuda.synchronize()
    assert handle.sgemm_cube_check()[0] == 0
    handle.destroy()


def parts(act, z):
    """Value, slope, the slope's two terms, and the relative error of the weight (Phi or a sigmoid)."""
    if act == ACT_GELU:
        w = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        bell = torch.exp(-z * z / 2) / math.sqrt(2.0 * math.pi)
        return z * w, w + z * bell, w.abs() + (z * bell).abs(), (24 + 5 * z * z / 2) * U
    if act == ACT_SILU:
        a, da = z, torch.ones_like(z)
    else:
        a, da = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3), 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    w = torch.sigmoid(a)
    second = z * torch.sigmoid(-a) * w * da
    return z * w, w + second, w + second.abs(), (12 + 3 * a.abs()) * U


@pytest.mark.parametrize("act,low", [(ACT_GELU, -8.0), (ACT_GELU_TANH, -6.0), (ACT_SILU, -60.0)])
@pytest.mark.parametrize("m", [1, 3, 24, 300])
def test_values(h, act, low, m):
    n, k = 4096, 4
    x, w = torch.ones(m, k, device=DEV), torch.zeros(k, n, device=DEV)
    bias = torch.cat([torch.linspace(low, 10.0, n - 1024, device=DEV), torch.linspace(-0.01, 0.01, 1024, device=DEV)])
    y, z = torch.empty(m, n, device=DEV), torch.empty(m, n, device=DEV)
    h.sgemm_cube_linear(x, w, y, bias=bias, activation=act, preact=z, weight_layout=WEIGHT_KN)
    assert torch.equal(z, bias.expand(m, n))
    want, _, _, rel = parts(act, z.double())
    over = (y.double() - want).abs() - (rel + 2 * U) * want.abs()
    assert bool((over <= 2.0 ** -126).all()), (float(over.max()), float(z.flatten()[over.argmax()]))


@pytest.mark.parametrize("act,low", [(ACT_GELU, -8.0), (ACT_GELU_TANH, -6.0), (ACT_SILU, -60.0)])
def test_slopes(h, act, low):
    n = 1 << 16
    z = torch.linspace(low, 10.0, n, device=DEV)[None].contiguous()
    dy, db = torch.ones(1, n, device=DEV), torch.empty(n, device=DEV)
    x, w = torch.ones(1, 1, device=DEV), torch.zeros(1, n, device=DEV)
    h.sgemm_cube_linear_backward(dy, x, w, dbias=db, preact=z, activation=act)
    _, want, size, rel = parts(act, z[0].double())
    over = (db.double() - want).abs() - (rel + 6 * U) * size
    assert bool((over <= 2.0 ** -126).all()), (float(over.max()), float(z[0, over.argmax()]))
