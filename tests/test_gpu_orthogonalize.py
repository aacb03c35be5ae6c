"""Newton-Schulz orthogonalisation against the polynomial in 64 bits.

Bounds, in the Frobenius norm, with |X0| = 1.  e = (8 + d / 128) 2^-23 + 2^-20 is what a product of depth d and the two words of
its factors and of its result are off by.  One step with a, b, c = 3.4445, -4.775, 2.0315:  |dA| <= 2 e,
|dP| <= 4.775 * 2 e + 2.0315 * 3 e, |dO| <= |dP| + 3.4445 * 2 e, 23 e in all, of a result that is at least |f(1)| = 0.7 in the
norm: 33 e.  A further step passes on what it finds with a factor of at most max |f'| <= 4 (singular values up to 1.21) and
adds its own.  FP32 products err alike, so over several steps the result is also held to eight times what plain FP32 makes of it."""
import pytest
import torch

from paper_2507_23387_b200 import binding
from paper_2507_23387_b200.binding import INVALID_ARG

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
QUINTIC = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    torch.cuda.synchronize()
    assert handle.sgemm_cube_check()[0] == 0
    handle.destroy()


def rand(seed, *shape, scale=1.0):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV) * scale


def steps_of(g, dtype, steps, coefficients=None, eps=1e-7):
    """X after `steps` steps, all of it in `dtype`."""
    x = g.to(dtype)
    x = x / (g.double().norm() + eps).to(dtype)
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    for i in range(steps):
        a, b, c = QUINTIC if coefficients is None else coefficients[i]
        m = x @ x.t()
        x = a * x + (b * m + c * (m @ m)) @ x
    return x.t() if tall else x


def bound(rows, cols, steps):
    e = (8 + max(rows, cols) / 128) * 2.0 ** -23 + 2.0 ** -20
    return 33 * e * (4 ** steps - 1) / 3


def check(h, g, steps, got=None, coefficients=None, **kw):
    want = steps_of(g, torch.float64, steps, coefficients)
    if got is None:
        got = torch.full(g.shape, float("nan"), device=DEV)
        h.sgemm_cube_orthogonalize(g, got, steps=steps, coefficients=coefficients, **kw)
    err, norm = float((got.double() - want).norm()), float(want.norm())
    assert err <= bound(*g.shape, steps) * norm, (err / norm, bound(*g.shape, steps))
    plain = float((steps_of(g, torch.float32, steps, coefficients).double() - want).norm())
    assert err <= 8 * plain + bound(*g.shape, 1) * norm, (err / norm, plain / norm)
    return got


# one entry, vectors, odd sizes on both sides of words, tiles and pairs; tiles of a triangle with and without a shared k range
SIZES = [(1, 1), (1, 50), (50, 1), (7, 5), (64, 64), (100, 129), (129, 100), (127, 300), (257, 700), (700, 257), (300, 300), (513, 1030),
         (1030, 513), (2100, 2300), (2300, 2100)]


@pytest.mark.parametrize("steps", [1, 2, 5])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_steps(h, rows, cols, steps):
    g = rand(rows * 7 + cols, rows, cols, scale=0.01)
    first = check(h, g, steps)
    assert torch.equal(first, check(h, g, steps))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(24, 40), (131, 77), (300, 1000)])
def test_16_bit_gradients(h, dtype, rows, cols):
    check(h, rand(1, rows, cols).to(dtype), 1)
    check(h, rand(2, rows, cols).to(dtype), 5)


@pytest.mark.parametrize("pair", [0, 1])
@pytest.mark.parametrize("split", [0, 1])
@pytest.mark.parametrize("rows,cols", [(390, 1100), (1100, 390), (640, 640)])
def test_kernel_variants(pair, split, rows, cols):
    h = binding.Handle(0)
    h.sgemm_cube_set_option(binding.OPT_CTA_PAIR, pair)
    h.sgemm_cube_set_option(binding.OPT_SPLIT_K, split)
    check(h, rand(3, rows, cols), 1)
    check(h, rand(4, rows, cols), 3)
    assert h.sgemm_cube_check()[0] == 0
    h.destroy()


def test_result_has_nearly_orthonormal_rows(h):
    """The published coefficients bring singular values from 0.02 on into [0.67, 1.21]."""
    for shape in ((200, 500), (500, 200)):
        o = check(h, rand(5, *shape), 5)
        s = torch.linalg.svdvals(o.double())
        assert float(s.min()) > 0.6 and float(s.max()) < 1.25


@pytest.mark.parametrize("scale", [1e-30, 1e-38, 1e30, 3e37])
def test_gradients_of_any_size(h, scale):
    g = rand(6, 100, 140).mul_(scale)
    if scale < 1e-35:
        g[::2] *= 1e-4                                       # subnormal entries
    got = torch.empty(100, 140, device=DEV)
    h.sgemm_cube_orthogonalize(g, got, steps=1, eps=0.0)
    check(h, (g.double() / g.double().abs().max()).float(), 1, got=got)


def test_coefficients_of_every_step(h):
    cubic = [(1.5, -0.5, 0.0)] * 3
    check(h, rand(7, 90, 140), 3, coefficients=cubic)
    mixed = [(4.0, -6.0, 2.9), (2.5, -2.0, 0.7), (1.875, -1.25, 0.375)]
    check(h, rand(8, 140, 90), 3, coefficients=mixed)
    same = torch.empty(90, 140, device=DEV)
    other = torch.empty(90, 140, device=DEV)
    g = rand(9, 90, 140)
    h.sgemm_cube_orthogonalize(g, same, steps=4, coefficients=QUINTIC)
    h.sgemm_cube_orthogonalize(g, other, steps=4)
    assert torch.equal(same, other)


@pytest.mark.parametrize("rows,cols", [(70, 130), (130, 70), (300, 520)])
def test_scaled_and_added_in_place(h, rows, cols):
    g, r = rand(10, rows, cols), rand(11, rows, cols)
    x = check(h, g, 2)
    out = torch.empty_like(g)
    h.sgemm_cube_orthogonalize(g, out, steps=2, scale=-0.3, residual=r, beta=0.9)
    want = -0.3 * x.double() + 0.9 * r.double()
    # the scale is taken into the product's way back: a rounding of each term and one of the sum
    assert bool(((out.double() - want).abs() <= 4 * 2.0 ** -24 * (0.3 * x.double().abs() + 0.9 * r.double().abs())).all())
    held = r.clone()
    h.sgemm_cube_orthogonalize(g, held, steps=2, scale=-0.3, residual=held, beta=0.9)
    assert torch.equal(held, out)
    own = g.clone()
    h.sgemm_cube_orthogonalize(own, own, steps=2)
    assert torch.equal(own, x)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ld,ldo,off", [(90, 91, 0), (93, 96, 3), (96, 90, 1)])
def test_strides_and_any_alignment(h, dtype, ld, ldo, off):
    rows, cols = 45, 90
    buf = torch.full((rows * ld + off,), float("nan"), device=DEV, dtype=dtype)
    g = torch.as_strided(buf, (rows, cols), (ld, 1), off)
    g.copy_(rand(12, rows, cols))
    room = torch.full((rows * ldo + off,), float("nan"), device=DEV)
    o = torch.as_strided(room, (rows, cols), (ldo, 1), off)
    h.sgemm_cube_orthogonalize(g, o, steps=2)
    plain = torch.empty(rows, cols, device=DEV)
    h.sgemm_cube_orthogonalize(g.contiguous(), plain, steps=2)
    assert torch.equal(o, plain)
    check(h, g, 2, got=plain)
    inside = torch.zeros_like(room, dtype=torch.bool)
    torch.as_strided(inside, (rows, cols), (ldo, 1), off).fill_(True)
    assert bool(torch.isnan(room[~inside]).all())


def test_zeros_and_values_that_are_not_finite(h):
    o = torch.full((30, 50), float("nan"), device=DEV)
    for eps in (0.0, 1e-7):
        h.sgemm_cube_orthogonalize(torch.zeros(30, 50, device=DEV), o, eps=eps)
        assert not o.any()
    for bad in (float("nan"), float("inf")):
        g = rand(13, 30, 50)
        g[4, 5] = bad
        h.sgemm_cube_orthogonalize(g, o)
        assert bool(torch.isnan(o).all())
    # one direction only: f(1) in every step
    g = torch.zeros(30, 50, device=DEV)
    g[3, 7] = 2.0
    check(h, g, 5)


def test_nothing_to_do(h):
    for shape in ((0, 5), (5, 0)):
        h.sgemm_cube_orthogonalize(torch.empty(shape, device=DEV), torch.empty(shape, device=DEV))


def test_refusals(h):
    lib, rows, cols = binding.load(), 6, 10
    g, o, r = rand(14, rows, cols), rand(15, rows, cols), rand(16, rows, cols)
    f = __import__("ctypes").c_float

    def call(rows=rows, cols=cols, dtype=0, g=g.data_ptr(), ldg=cols, steps=2, k=None, eps=1e-7, scale=1.0, r=r.data_ptr(), ldr=cols, beta=1.0,
             o=o.data_ptr(), ldo=cols):
        return lib.sgemm_cube_orthogonalize(h._h, rows, cols, dtype, g, ldg, steps, k, eps, scale, r, ldr, beta, o, ldo, None)

    assert call() == 0 and call(r=None) == 0 and call(r=o.data_ptr()) == 0 and call(o=g.data_ptr()) == 0
    assert call(rows=1, o=g.data_ptr(), ldo=cols + 1) == 0         # one row has no leading dimension
    before = h.sgemm_cube_launch_count()
    nan = float("nan")
    for bad in (dict(rows=-1), dict(cols=2 ** 31 - 1), dict(dtype=3), dict(g=None), dict(o=None), dict(g=g.data_ptr() + 2), dict(o=o.data_ptr() + 1),
                dict(r=r.data_ptr() + 2), dict(ldg=cols - 1), dict(ldo=cols - 1), dict(ldr=cols - 1), dict(steps=0), dict(steps=65), dict(eps=-1.0),
                dict(eps=nan), dict(scale=nan), dict(beta=float("inf")), dict(r=o.data_ptr(), ldo=cols + 1), dict(o=g.data_ptr(), ldo=cols + 1), dict(o=g.data_ptr(), dtype=1),
                dict(k=(f * 6)(1, 0, 0, nan, 0, 0)), dict(k=(f * 6)(0, 0, 0, 1, 0, 0)), dict(k=(f * 6)(2000, 0, 0, 2000, 0, 0))):
        assert call(**bad) == INVALID_ARG, bad
    assert h.sgemm_cube_launch_count() == before
