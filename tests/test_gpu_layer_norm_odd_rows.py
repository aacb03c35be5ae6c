"""Gradients of the layer norm over rows that start anywhere between two 16-byte boundaries: more rows than are worked on
at once, every start, neighbours of NaN, tensors that agree in where rows start and tensors that do not.
Tolerances: those of the layer norm's own tests."""
import pytest
import torch

from paper_2507_23387_b200 import binding
from test_gpu_layer_norm import DEV, TYPES, check_backward, pitched, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    torch.cuda.synchronize()
    handle.destroy()


def gradients(h, dy, x, w, out=None):
    rows, cols = x.shape
    mean, rstd = x.double().mean(1).float(), (1 / torch.sqrt(x.double().var(1, unbiased=False) + 1e-5)).float()
    out = torch.empty_like(x) if out is None else out
    dw, db = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    h.sgemm_cube_layer_norm_backward(dy, x, mean, rstd, out, weight=w, dweight=dw, dbias=db)
    return out, dw, db, mean, rstd


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(20000, 9), (9000, 131), (6000, 505), (5001, 1001), (3000, 2041), (2500, 4090), (900, 7001),
                                       (500, 9999), (400, 16377), (300, 16383)])
def test_many_odd_rows(h, rows, cols, dtype):
    x, dy, w = rand(1, rows, cols, shift=0.5, dtype=dtype), rand(2, rows, cols, dtype=dtype), rand(3, cols)
    dx, dw, db, mean, rstd = gradients(h, dy, x, w)
    check_backward(dx, dw, db, dy, x, w, mean, rstd)
    again = gradients(h, dy, x, w)
    assert all(torch.equal(a, b) for a, b in zip(again[:3], (dx, dw, db)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [64, 67, 1003])
def test_every_start(h, cols, dtype):
    """Leading dimensions and offsets of all residues, alike for all tensors, then different ones."""
    rows = 41
    x, dy, w = rand(4, rows, cols, dtype=dtype), rand(5, rows, cols, dtype=dtype), rand(6, cols)
    for offset in range(8):
        for extra in (0, 1, 2, 5):
            out = pitched(torch.zeros_like(x), extra, offset)
            dx, dw, db, mean, rstd = gradients(h, pitched(dy, extra, offset), pitched(x, extra, offset), w, out)
            check_backward(dx, dw, db, dy, x, w, mean, rstd)
            assert int(torch.isnan(out._base.view(-1)).sum()) == offset + rows * extra
    for places in (((1, 0), (0, 0), (0, 0)), ((0, 1), (0, 1), (0, 2)), ((3, 2), (3, 2), (4, 2))):
        (ex, ox), (eg, og), (eo, oo) = places
        out = pitched(torch.zeros_like(x), eo, oo)
        dx, dw, db, mean, rstd = gradients(h, pitched(dy, eg, og), pitched(x, ex, ox), w, out)
        check_backward(dx, dw, db, dy, x, w, mean, rstd)


@pytest.mark.parametrize("dtype", TYPES)
def test_nan_stays_in_its_row(h, dtype):
    rows, cols = 700, 1005
    x, dy, w = rand(7, rows, cols, dtype=dtype), rand(8, rows, cols, dtype=dtype), rand(9, cols)
    want = gradients(h, dy, x, w)[0]
    bad = torch.arange(rows, device=DEV) % 3 == 0
    x[bad], dy[bad] = float("nan"), float("inf")
    got = gradients(h, dy, x, w)[0]
    assert torch.equal(got[~bad], want[~bad]) and not torch.isfinite(got[bad]).any()


def test_in_place_and_one_row(h):
    for rows, cols in ((1, 77), (2, 1001), (2000, 1001)):
        x, dy, w = rand(10, rows, cols), rand(11, rows, cols), rand(12, cols)
        want = gradients(h, dy, x, w)
        got = gradients(h, dy, x, w, out=dy)
        assert all(torch.equal(a, b) for a, b in zip(got[:3], want[:3]))
