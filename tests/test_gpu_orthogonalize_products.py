"""Orthogonalised updates that take a launch for every product, against the polynomial in 64 bits: matrices above the size up to
which all products are one launch.  Tiles of a triangle and their mirror images, as single blocks and pairs, whole and cut along k;
wide, tall and square, odd sizes, 16-bit gradients, results on odd addresses, in place.

Bounds: those of the smaller updates; they depend on the depth of the products alone."""
import pytest
import torch

from paper_2507_23387_b200 import binding
from test_gpu_orthogonalize import DEV, check, h, rand  # noqa: F401  (h: the handle's fixture)

pytestmark = pytest.mark.gpu

# square, wide and tall; few tiles of a triangle under long sums, which are cut along k
SIZES = [(2301, 2500), (2500, 2301), (2600, 2600), (641, 30001), (30001, 641)]


def counted(handle, steps, call):
    """The call's launches: the sum of squares, the first words, and three products a step."""
    before = handle.sgemm_cube_launch_count()
    result = call()
    assert handle.sgemm_cube_launch_count() - before == 2 + 3 * steps
    return result


@pytest.mark.parametrize("steps", [1, 2, 5])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_steps(h, rows, cols, steps):  # noqa: F811
    g = rand(rows + cols, rows, cols, scale=0.01)
    first = counted(h, steps, lambda: check(h, g, steps))
    assert torch.equal(first, check(h, g, steps))


# (1500 rows: 42 tiles of the triangle, which leave more than half of the SMs idle)
@pytest.mark.parametrize("pair", [0, 1, 2])
@pytest.mark.parametrize("split", [0, 1])
@pytest.mark.parametrize("rows,cols", [(2301, 2500), (2500, 2301), (1500, 5401), (5401, 1500), (641, 30001)])
def test_kernel_variants(pair, split, rows, cols):
    handle = binding.Handle(0)
    handle.sgemm_cube_set_option(binding.OPT_CTA_PAIR, pair)
    handle.sgemm_cube_set_option(binding.OPT_SPLIT_K, split)
    counted(handle, 1, lambda: check(handle, rand(3, rows, cols), 1))
    check(handle, rand(4, rows, cols), 3)
    assert handle.sgemm_cube_check()[0] == 0
    handle.destroy()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(2303, 2400), (2400, 2303), (700, 25001)])
def test_16_bit_gradients(h, dtype, rows, cols):  # noqa: F811
    counted(h, 1, lambda: check(h, rand(5, rows, cols).to(dtype), 1))
    check(h, rand(6, rows, cols).to(dtype), 5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,pad,pado,off", [(2301, 2500, 0, 1, 0), (2500, 2301, 3, 7, 3), (2400, 2304, 8, 0, 1)])
def test_strides_and_any_alignment(h, dtype, rows, cols, pad, pado, off):  # noqa: F811
    ld, ldo = cols + pad, cols + pado
    buf = torch.full((rows * ld + off,), float("nan"), device=DEV, dtype=dtype)
    g = torch.as_strided(buf, (rows, cols), (ld, 1), off)
    g.copy_(rand(7, rows, cols))
    room = torch.full((rows * ldo + off,), float("nan"), device=DEV)
    o = torch.as_strided(room, (rows, cols), (ldo, 1), off)
    counted(h, 2, lambda: h.sgemm_cube_orthogonalize(g, o, steps=2))
    check(h, g, 2, got=o)
    plain = torch.empty(rows, cols, device=DEV)
    h.sgemm_cube_orthogonalize(g.contiguous(), plain, steps=2)
    # (the sum of squares is taken in another order where rows take no vectors: FP64, rounded to FP32 behind it)
    assert float((o.double() - plain.double()).norm()) <= 2.0 ** -20 * float(plain.double().norm())
    inside = torch.zeros_like(room, dtype=torch.bool)
    torch.as_strided(inside, (rows, cols), (ldo, 1), off).fill_(True)
    assert bool(torch.isnan(room[~inside]).all())


@pytest.mark.parametrize("rows,cols,ldr", [(2301, 2500, 2501), (2500, 2304, 2304)])
def test_scaled_and_added_in_place(h, rows, cols, ldr):  # noqa: F811
    g = rand(8, rows, cols)
    r = torch.as_strided(torch.empty(rows * ldr, device=DEV), (rows, cols), (ldr, 1))
    r.copy_(rand(9, rows, cols))
    x = check(h, g, 2)
    out = torch.empty_like(g)
    counted(h, 2, lambda: h.sgemm_cube_orthogonalize(g, out, steps=2, scale=-0.3, residual=r, beta=0.9))
    want = -0.3 * x.double() + 0.9 * r.double()
    # the scale is taken into the product's way back: a rounding of each term and one of the sum
    assert bool(((out.double() - want).abs() <= 4 * 2.0 ** -24 * (0.3 * x.double().abs() + 0.9 * r.double().abs())).all())
    h.sgemm_cube_orthogonalize(g, r, steps=2, scale=-0.3, residual=r, beta=0.9)
    assert torch.equal(r, out)
    h.sgemm_cube_orthogonalize(g, g, steps=2)
    assert torch.equal(g, x)


@pytest.mark.parametrize("rows,cols", [(2301, 2500), (2500, 2301)])
def test_zeros_and_values_that_are_not_finite(h, rows, cols):  # noqa: F811
    g, o = torch.zeros(rows, cols, device=DEV), torch.full((rows, cols), float("nan"), device=DEV)
    for eps in (0.0, 1e-7):
        h.sgemm_cube_orthogonalize(g, o, eps=eps)
        assert not o.any()
    for bad in (float("nan"), float("inf")):
        g = rand(10, rows, cols)
        g[rows - 1, cols - 1] = bad
        h.sgemm_cube_orthogonalize(g, o)
        assert bool(torch.isnan(o).all())
    for scale in (1e-38, 3e37):
        g = rand(11, rows, cols).mul_(scale)
        h.sgemm_cube_orthogonalize(g, o, steps=1, eps=0.0)
        check(h, (g.double() / g.double().abs().max()).float(), 1, got=o)


def test_captured_and_replayed_on_other_gradients():
    handle = binding.Handle(0)
    g, o = rand(12, 2301, 2500), torch.empty(2301, 2500, device=DEV)
    handle.sgemm_cube_orthogonalize(g, o, steps=2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        handle.sgemm_cube_orthogonalize(g, o, steps=2)
    for seed in (13, 14):
        g.copy_(rand(seed, 2301, 2500))
        o.fill_(float("nan"))
        graph.replay()
        check(handle, g, 2, got=o)
    assert handle.sgemm_cube_check()[0] == 0
    del graph
    handle.destroy()
