"""Layer normalisation of rows whose mean is far above their spread, and of constant rows, against FP64.

Tolerances (u = 2^-24).  On any path a row's sums add at most D = 64 + cols / 1024 numbers one after the other (a
thread's own, then trees over a warp and over the warps).  The first mean is off by e0 <= D u mean|x|; it is
corrected by the average c of the differences d = x - m0, which is off by D u mean|d| with
mean|d| <= mean|x - mean| + e0.  What is left in the centred value is that, and one rounding of d and of c: it does not
grow with the offset but through e0, which counts only once more multiplied by u.  The variance is off by
D u of itself and of 2 e0^2."""
import pytest
import torch

from paper_2507_23387_b200 import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DEV = "cuda:0"
ROUND = {torch.float32: U, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.float32, torch.float16, torch.bfloat16]
# part of a warp, every number of warps a row, aligned and odd, longer than a block holds
COLS = [3, 31, 282, 307, 512, 1000, 2047, 3000, 4096, 4100, 8193, 12345, 16384, 16385, 33000]


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    torch.cuda.synchronize()
    handle.destroy()


def check(h, x, eps=1e-5, w=None, b=None):
    rows, cols = x.shape
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    h.sgemm_cube_layer_norm(x, y, weight=w, bias=b, eps=eps, mean=mean, rstd=rstd)
    xd, D = x.double(), 64 + cols / 1024
    m = xd.mean(1, keepdim=True)
    var = ((xd - m) ** 2).mean(1, keepdim=True)
    r = 1 / torch.sqrt(var + torch.tensor(eps, dtype=torch.float32).double().item())
    n = (xd - m) * r
    wd = torch.ones(cols, device=DEV, dtype=torch.float64) if w is None else w.double()
    bd = torch.zeros(cols, device=DEV, dtype=torch.float64) if b is None else b.double()
    want = n * wd + bd
    e0 = D * U * xd.abs().mean(1, keepdim=True)
    spread = (xd - m).abs().mean(1, keepdim=True)
    e_c = (D + 3) * U * (spread + e0)
    e_d = U * ((xd - m).abs() + e0) + e_c
    e_r = (D + 3) * U * (1 + 2 * e0 ** 2 * r ** 2) + 4 * U
    tol = (e_d * r + n.abs() * e_r + 3 * U * n.abs()) * wd.abs() + U * want.abs() + ROUND[x.dtype] * want.abs()
    tol = tol + (2.0 ** -25 if x.dtype == torch.float16 else 2.0 ** -126)
    assert torch.isfinite(y).all()
    assert bool(((y.double() - want).abs() <= tol).all()), float(((y.double() - want).abs() - tol).max())
    assert bool(((mean.double()[:, None] - m).abs() <= U * m.abs() + e_c).all())
    assert bool(((rstd.double()[:, None] / r - 1).abs() <= e_r).all())
    return y, mean


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_constant_rows(h, cols, dtype):
    values = torch.tensor([3.0, 7.0, 1000.0, -0.1, 30000.0, 1.0 / 3.0], device=DEV).to(dtype)
    x = values[:, None].expand(-1, cols).contiguous()
    y, mean = check(h, x)
    assert torch.equal(mean, values.float())                  # the correction leaves less than half a unit
    assert float(y.float().abs().max()) <= 1e-3
    b = torch.linspace(-1, 1, cols, device=DEV)
    check(h, x, b=b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_rows_far_from_zero(h, cols, dtype):
    g = torch.Generator(device=DEV).manual_seed(cols)
    at = torch.tensor([0.0, 10.0, 1000.0, -1000.0, 1e4, 3e4, 0.5], device=DEV)[:, None]
    x = (torch.randn((7, cols), generator=g, device=DEV) + at).to(dtype)
    w, b = torch.randn(cols, generator=g, device=DEV), torch.randn(cols, generator=g, device=DEV)
    check(h, x)
    check(h, x, w=w, b=b)
    check(h, x, eps=0.0) if dtype == torch.float32 and cols > 31 else None


@pytest.mark.parametrize("cols", [282, 4096, 5001, 20000])
def test_a_column_that_stands_out(h, cols):
    """One large entry moves the mean far from every other entry; many rows, so that blocks take several."""
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn((1500, cols), generator=g, device=DEV)
    x[:, 17] = 1e6
    check(h, x)
    x = torch.randn((1500, cols), generator=g, device=DEV) * 1e-3 + 100.0
    check(h, x, eps=1e-12)


def test_nonfinite_rows_stay_by_themselves(h):
    for cols in (300, 4099, 20000):
        x = torch.ones(5, cols, device=DEV) * 1000
        x[1, 3], x[3, cols - 1] = float("nan"), float("inf")
        y = torch.empty_like(x)
        h.sgemm_cube_layer_norm(x, y)
        assert torch.isnan(y[[1, 3]]).all() and float(y[[0, 2, 4]].abs().max()) <= 1e-3
