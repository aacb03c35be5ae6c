"""Packing a matrix that is too large for one launch: the words and the exponent do not depend on where it lies, nor on which element is
the largest."""
import pytest
import torch

from paper_2507_23387_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    torch.cuda.synchronize()
    assert handle.sgemm_cube_check()[0] == 0
    handle.destroy()


def packed(h, x):
    w = binding.PackedMatrix(*x.shape, device=DEV)
    w.hi.fill_(float("nan"))
    w.lo.fill_(float("nan"))
    h.sgemm_cube_pack(x, w)
    return w


# Rows of 4001 and 9 behind one another or apart, of 4000 where nothing is odd but the address, a few very long ones
@pytest.mark.parametrize("rows,cols,ld", [(5003, 4001, 4001), (5003, 4000, 4000), (5003, 4001, 4003), (2000003, 9, 9), (7, 3000001, 3000001),
                                          (3000001, 7, 7)])
@pytest.mark.parametrize("off", [0, 1, 2, 3, 4])
@pytest.mark.parametrize("largest", [0, 2, -1])
def test_words_of_any_address(h, rows, cols, ld, off, largest):
    g = torch.Generator(device=DEV).manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=g, device=DEV)
    x.view(-1)[largest] = 1000.0
    wide = (cols + 3) // 4 * 4
    even = torch.zeros(rows, wide, device=DEV)[:, :cols]
    even.copy_(x)
    buf = torch.full((off + (rows - 1) * ld + cols + 16,), float("inf"), device=DEV)
    odd = torch.as_strided(buf, (rows, cols), (ld, 1), off)
    odd.copy_(x)
    a, b = packed(h, odd), packed(h, even)
    assert a.exp.item() == b.exp.item() == 15 - 9                    # 1000 lies in the binade of 2^9
    assert torch.equal(a.hi.view(torch.int16), b.hi.view(torch.int16))
    assert torch.equal(a.lo.view(torch.int16), b.lo.view(torch.int16))
    # 22 bits and more of each element's value
    back = (a.hi[:, :cols].double() + a.lo[:, :cols].double() / 2048) * 2.0 ** -6
    assert bool(((back - x.double()).abs() <= 2.0 ** -22 * x.double().abs() + 2.0 ** -41).all())
