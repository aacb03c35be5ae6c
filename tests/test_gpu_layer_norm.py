"""Layer normalisation and its gradients against the definition in FP64.

Tolerances (u = 2^-24, t the element type's unit roundoff).  A row's sums add at most `depth` = 96 + cols / 256
numbers one after the other on any path (a thread's own, then trees), so mean is off by depth u mean|x| and the
statistics by 2 depth u; the elementwise steps add a few u.  Everything below is that, written out."""
import pytest
import torch

from paper_2507_23387_b200 import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DEV = "cuda:0"
ROUND = {torch.float32: U, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    torch.cuda.synchronize()
    handle.destroy()


def rand(seed, *shape, scale=1.0, shift=0.0, dtype=torch.float32):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale + shift).to(dtype)


def pitched(t, extra, offset=0):
    r, c = t.shape
    buf = torch.full((r * (c + extra) + offset,), float("nan"), device=t.device, dtype=t.dtype)
    v = buf[offset:offset + r * (c + extra)].view(r, c + extra)[:, :c]
    v.copy_(t)
    return v


def norm64(x, w, b, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    n = (x - mean) * rstd
    y = n * (1 if w is None else w.double()) + (0 if b is None else b.double())
    return y, n, mean, rstd


def depth(cols):
    return 96 + cols / 256


def check_forward(y, mean, rstd, x, w, b, eps):
    want, n, m64, r64 = norm64(x, w, b, eps)
    d, wa = depth(x.shape[1]), 1.0 if w is None else w.double().abs()
    size = x.double().abs().mean(1, keepdim=True)
    e_mean = d * U * size
    # the mean's error moves n by e_mean rstd and enters the variance squared
    e_n = e_mean * r64 + n.abs() * (2 * d * U + (e_mean * r64) ** 2) + 4 * U * (n.abs() + x.double().abs() * r64)
    tol = e_n * wa + 2 * U * want.abs() + ROUND[x.dtype] * want.abs() + (2.0 ** -25 if x.dtype == torch.float16 else 0)
    assert torch.isfinite(y).all()
    assert bool(((y.double() - want).abs() <= tol).all())
    if mean is not None:
        assert bool(((mean.double() - m64[:, 0]).abs() <= e_mean[:, 0] + 2 * U * m64[:, 0].abs()).all())
        assert bool(((rstd / r64[:, 0] - 1).abs() <= 2 * d * U + (e_mean * r64)[:, 0] ** 2 + 4 * U).all())


# one column, part of a warp, each number of warps a row, their limits and one past, odd, longer than a block holds
COLS = [1, 2, 5, 31, 128, 129, 512, 513, 1000, 1024, 1025, 2047, 2048, 4096, 4100, 8192, 8200, 16384, 16400, 33000]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_forward(h, cols, dtype):
    for rows in (1, 3, 37):
        x = rand(cols, rows, cols, scale=2.0, shift=0.7, dtype=dtype)
        w, b = rand(1, cols, shift=1.0), rand(2, cols)
        y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        h.sgemm_cube_layer_norm(x, y, weight=w, bias=b, eps=1e-5, mean=mean, rstd=rstd)
        check_forward(y, mean, rstd, x, w, b, 1e-5)


@pytest.mark.parametrize("dtype", TYPES)
def test_forward_options_strides_in_place(h, dtype):
    for rows, cols in ((5, 64), (9, 1030), (4, 5000)):
        x = rand(3, rows, cols, dtype=dtype)
        w, b = rand(4, cols), rand(5, cols)
        for extra, offset in ((0, 0), (8, 0), (3, 0), (1, 1), (16, 5)):
            for ww, bb in ((w, None), (None, b), (None, None)):
                out = pitched(torch.zeros_like(x), extra, offset)
                h.sgemm_cube_layer_norm(pitched(x, extra, offset), out, weight=ww, bias=bb, eps=1e-6)
                check_forward(out, None, None, x, ww, bb, 1e-6)
                assert torch.isnan(out._base.view(-1)).sum() == offset + rows * extra
        y = torch.empty_like(x)
        h.sgemm_cube_layer_norm(x, y, weight=w, bias=b)
        inplace = x.clone()
        h.sgemm_cube_layer_norm(inplace, inplace, weight=w, bias=b)
        assert torch.equal(inplace, y)


def test_forward_hard_rows(h):
    """A mean far above the spread, constant rows, zero rows, huge rows, and a NaN that stays in its row."""
    cols = 3000
    x = rand(6, 6, cols)
    x[0] += 1000.0
    x[1] = 3.0
    x[2] = 0.0
    x[3] *= 1e15
    x[4, 7] = float("nan")
    y = torch.empty_like(x)
    h.sgemm_cube_layer_norm(x, y, eps=1e-5)
    keep = [0, 1, 2, 3, 5]
    check_forward(y[keep], None, None, x[keep], None, None, 1e-5)
    assert torch.isnan(y[4]).all()


def check_backward(dx, dw, db, dy, x, w, mean, rstd):
    rows, cols = x.shape
    g, xd = dy.double(), x.double()
    n = (xd - mean.double()[:, None]) * rstd.double()[:, None]          # the statistics are inputs here
    wd = torch.ones(cols, device=DEV, dtype=torch.float64) if w is None else w.double()
    u = g * wd
    mu, mun = u.mean(1, keepdim=True), (u * n).mean(1, keepdim=True)
    e_n = 3 * U * (n.abs() + xd.abs() * rstd.double()[:, None])
    if dx is not None:
        want = rstd.double()[:, None] * (u - mu - n * mun)
        d = depth(cols)
        au, aun = u.abs().mean(1, keepdim=True), (u.abs() * (n.abs() + e_n)).mean(1, keepdim=True)
        e_mun = d * U * aun + (u.abs() * e_n).mean(1, keepdim=True)
        tol = rstd.double()[:, None] * (3 * U * u.abs() + d * U * au + n.abs() * e_mun + e_n * aun + 4 * U * (au + n.abs() * aun))
        tol = tol + ROUND[x.dtype] * want.abs() + (2.0 ** -25 if x.dtype == torch.float16 else 0)
        assert torch.isfinite(dx).all()
        assert bool(((dx.double() - want).abs() <= tol).all())
    if dw is not None:
        tol = (rows + 4) * U * (g * n).abs().sum(0) + (g.abs() * e_n).sum(0)
        assert bool(((dw.double() - (g * n).sum(0)).abs() <= tol).all())
    if db is not None:
        assert bool(((db.double() - g.sum(0)).abs() <= (rows + 2) * U * g.abs().sum(0)).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_backward(h, cols, dtype):
    for rows in (1, 5, 700 if cols <= 2048 else 170):
        x, dy = rand(cols, rows, cols, scale=2.0, shift=0.5, dtype=dtype), rand(7, rows, cols, scale=0.1, dtype=dtype)
        w = rand(8, cols, shift=1.0)
        y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        h.sgemm_cube_layer_norm(x, y, weight=w, mean=mean, rstd=rstd)
        dx, dw, db = torch.empty_like(x), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
        h.sgemm_cube_layer_norm_backward(dy, x, mean, rstd, dx, weight=w, dweight=dw, dbias=db)
        check_backward(dx, dw, db, dy, x, w, mean, rstd)


@pytest.mark.parametrize("dtype", TYPES)
def test_backward_options_strides_in_place(h, dtype):
    for rows, cols in ((50, 64), (33, 777), (20, 20000)):
        x, dy, w = rand(9, rows, cols, dtype=dtype), rand(10, rows, cols, dtype=dtype), rand(11, cols)
        mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        h.sgemm_cube_layer_norm(x, torch.empty_like(x), mean=mean, rstd=rstd)
        dx, dw, db = torch.empty_like(x), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
        h.sgemm_cube_layer_norm_backward(dy, x, mean, rstd, dx, weight=w, dweight=dw, dbias=db)
        check_backward(dx, dw, db, dy, x, w, mean, rstd)
        for extra, offset in ((8, 0), (1, 3)):
            out, dw2 = pitched(torch.zeros_like(x), extra, offset), torch.empty(cols, device=DEV)
            h.sgemm_cube_layer_norm_backward(pitched(dy, extra, offset), pitched(x, extra, offset), mean, rstd, out, dweight=dw2)
            check_backward(out, dw2, None, dy, x, None, mean, rstd)
            assert torch.isnan(out._base.view(-1)).sum() == offset + rows * extra
        db2 = torch.empty(cols, device=DEV)
        h.sgemm_cube_layer_norm_backward(dy, x, mean, rstd, None, weight=w, dbias=db2)
        assert torch.equal(db2, db)
        for _ in range(2):                                  # in place, and the same bits every time
            inplace = dy.clone()
            dw2 = torch.empty(cols, device=DEV)
            h.sgemm_cube_layer_norm_backward(inplace, x, mean, rstd, inplace, weight=w, dweight=dw2, dbias=db2)
            assert torch.equal(inplace, dx) and torch.equal(dw2, dw) and torch.equal(db2, db)


def test_gradient_against_differences(h):
    """<gradient, v> against the change of the kernel's own output: truncation and FP32 noise are both below 1e-3
    of the gradient's size at a step of 2^-5."""
    rows, cols, e = 12, 200, 2.0 ** -5
    x, w, b, dy = rand(12, rows, cols, scale=2.0), rand(13, cols), rand(14, cols), rand(15, rows, cols)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    h.sgemm_cube_layer_norm(x, y, weight=w, bias=b, mean=mean, rstd=rstd)
    grads = [torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)]
    h.sgemm_cube_layer_norm_backward(dy, x, mean, rstd, grads[0], weight=w, dweight=grads[1], dbias=grads[2])
    for i, t in enumerate((x, w, b)):
        v = torch.sign(grads[i]) / t.numel() ** 0.5
        values = []
        for s in (e, -e):
            moved = [x, w, b]
            moved[i] = t + s * v
            h.sgemm_cube_layer_norm(moved[0], y, weight=moved[1], bias=moved[2])
            values.append((y.double() * dy.double()).sum())
        slope, want = (values[0] - values[1]) / (2 * e), (grads[i].double() * v.double()).sum()
        assert abs(slope - want) <= 2e-3 * want, (i, float(slope), float(want))


def test_empty_and_refusals(h):
    e = torch.empty(0, 16, device=DEV)
    v = torch.empty(0, device=DEV)
    h.sgemm_cube_layer_norm(e, torch.empty_like(e))
    dw, db = torch.ones(16, device=DEV), torch.ones(16, device=DEV)
    h.sgemm_cube_layer_norm_backward(e, e, v, v, torch.empty_like(e), dweight=dw, dbias=db)
    assert not dw.any() and not db.any()
    x, y, s = rand(16, 4, 16), torch.empty(4, 16, device=DEV), torch.ones(4, device=DEV)
    for call in (lambda: h.sgemm_cube_layer_norm(x, y, eps=-1.0), lambda: h.sgemm_cube_layer_norm(x, y, eps=float("nan")),
                 lambda: h.sgemm_cube_layer_norm(torch.empty(4, 0, device=DEV), torch.empty(4, 0, device=DEV)),
                 lambda: h.sgemm_cube_layer_norm_backward(x, x, None, s, y)):
        with pytest.raises(binding.SgemmCubeError) as err:
            call()
        assert err.value.status == binding.INVALID_ARG
    with pytest.raises(KeyError):
        h.sgemm_cube_layer_norm(x.double(), y.double())
    with pytest.raises(AssertionError):
        h.sgemm_cube_layer_norm(x, y, weight=torch.ones(15, device=DEV))
    lib, p = binding.load(), x.data_ptr()
    bad = binding.INVALID_ARG
    assert lib.sgemm_cube_layer_norm(h._h, 4, 16, 3, p, 16, None, None, 0.0, y.data_ptr(), 16, None, None, None) == bad
    assert lib.sgemm_cube_layer_norm(h._h, 4, 16, 0, p, 15, None, None, 0.0, y.data_ptr(), 16, None, None, None) == bad
    assert lib.sgemm_cube_layer_norm(h._h, 4, 16, 0, p + 1, 16, None, None, 0.0, y.data_ptr(), 16, None, None, None) == bad
    assert lib.sgemm_cube_layer_norm(h._h, -1, 16, 0, p, 16, None, None, 0.0, y.data_ptr(), 16, None, None, None) == bad
    assert lib.sgemm_cube_layer_norm(None, 4, 16, 0, p, 16, None, None, 0.0, y.data_ptr(), 16, None, None, None) == bad
