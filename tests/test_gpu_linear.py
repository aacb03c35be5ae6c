"""The linear layer on the split product and its gradients, against the definition in FP64.

Tolerances (u = 2^-24).  Componentwise, a sum of K products on the tensor cores is off by at most
max(2K, K + 14) u times the sum of the magnitudes (truncating accumulation doubles the unit roundoff; for
short sums the two-word representation outweighs it).  That bound is loose for long sums, so the Frobenius
error is held to what the blocked summation can lose when partial sums stay near the result: 8 truncations
inside a 128-deep block, one addition per block, one ulp (2u) each, plus 2^-21 for words, activation and
epilogue.  Dropping a correction product would miss that by a factor of 30 or more.  Activations have
slopes of at most 1.2 and are themselves good to 2^-21 of (|z| + 1); slopes to 2^-20."""
import math

import numpy as np
import pytest
import torch

from paper_2507_23387_b200 import binding
from paper_2507_23387_b200.binding import (ACT_GELU, ACT_GELU_TANH, ACT_NONE, ACT_RELU, ACT_SILU, WEIGHT_KN, WEIGHT_NK,
                                           PackedMatrix)

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


def rand(seed, *shape, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV) * scale


def pitched(t, extra, offset=0):
    """The same values in a matrix with a longer leading dimension, `offset` elements past an aligned start."""
    r, c = t.shape
    buf = torch.full((r * (c + extra) + offset,), float("nan"), device=t.device, dtype=t.dtype)
    v = buf[offset:offset + r * (c + extra)].view(r, c + extra)[:, :c]
    v.copy_(t)
    return v


def act64(z, act):
    if act == ACT_RELU:
        return torch.relu(z)
    if act == ACT_GELU:
        return torch.nn.functional.gelu(z)
    if act == ACT_GELU_TANH:
        return torch.nn.functional.gelu(z, approximate="tanh")
    return torch.nn.functional.silu(z) if act == ACT_SILU else z


def slope64(z, act):
    z = z.clone().requires_grad_(True)
    with torch.enable_grad():
        return torch.autograd.grad(act64(z, act).sum(), z)[0]


def check_product(got, want, mag, depth, extra, label):
    err = (got.double() - want).abs()
    assert torch.isfinite(got).all(), label
    assert bool((err <= max(2 * depth, depth + 14) * U * 1.2 * mag + extra).all()), (label, float((err - extra).max()))
    frob = float(err.norm() / want.norm())
    assert frob <= (8 + depth / 128) * 2 * U + 2.0 ** -21, (label, frob)


def forward64(x, w, layout, bias):
    w = w.double().t() if layout == WEIGHT_NK else w.double()
    z, mag = x.double() @ w, x.double().abs() @ w.abs()
    if bias is not None:
        z, mag = z + bias.double(), mag + bias.double().abs()
    return z, mag


# few rows / tensor cores with one tile, several tiles, pairs; odd and ragged; k shorter and longer than a block
SHAPES = [(1, 1, 1), (1, 300, 517), (2, 129, 1024), (3, 40, 2048), (5, 257, 333), (8, 1000, 768), (9, 33, 65),
          (64, 512, 256), (128, 256, 128), (129, 255, 1000), (200, 700, 130), (300, 520, 1160), (512, 1536, 72)]


@pytest.mark.parametrize("layout", [WEIGHT_KN, WEIGHT_NK])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_forward(h, m, n, k, packed, layout):
    x, w = rand(1, m, k), rand(2, *((n, k) if layout == WEIGHT_NK else (k, n)), scale=k ** -0.5)
    bias, res = rand(3, n), rand(4, m, n)
    wo = w
    if packed:
        wo = PackedMatrix(*w.shape)
        h.sgemm_cube_pack(w, wo)
    y, z = torch.full((m, n), float("nan"), device=DEV), torch.full((m, n), float("nan"), device=DEV)
    h.sgemm_cube_linear(x, wo, y, bias=bias, residual=res, preact=z, weight_layout=layout)
    z64, mag = forward64(x, w, layout, bias)
    check_product(z, z64, mag, k, 0.0, "z")
    check_product(y, z64 + res.double(), mag, k, 2 * U * (z64.abs() + res.double().abs()), "y")


@pytest.mark.parametrize("act", [ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU])
@pytest.mark.parametrize("m", [4, 150])
def test_activations(h, m, act):
    n, k = 260, 320
    x, w = rand(5, m, k), rand(6, n, k, scale=3 * k ** -0.5)
    bias = torch.linspace(-30, 30, n, device=DEV)            # both tails of every activation
    y = torch.empty(m, n, device=DEV)
    h.sgemm_cube_linear(x, w, y, bias=bias, activation=act, weight_layout=WEIGHT_NK)
    z64, mag = forward64(x, w, WEIGHT_NK, bias)
    check_product(y, act64(z64, act), mag, k, 2.0 ** -21 * (z64.abs() + 1), "act %d" % act)


@pytest.mark.parametrize("m,n,k,layout", [(7, 96, 64, WEIGHT_KN), (7, 96, 64, WEIGHT_NK), (6, 101, 203, WEIGHT_KN),
                                          (6, 101, 203, WEIGHT_NK), (140, 99, 131, WEIGHT_KN), (140, 99, 131, WEIGHT_NK),
                                          (33, 64, 2500, WEIGHT_NK), (260, 300, 96, WEIGHT_KN)])
@pytest.mark.parametrize("extra,offset", [(0, 1), (3, 0), (4, 0), (5, 3)])
def test_strides_and_alignment(h, m, n, k, layout, extra, offset):
    x, w = rand(7, m, k), rand(8, *((n, k) if layout == WEIGHT_NK else (k, n)))
    bias, res = rand(9, n), rand(10, m, n)
    out = [pitched(torch.zeros(m, n, device=DEV), extra, offset) for _ in range(2)]
    h.sgemm_cube_linear(pitched(x, extra, offset), pitched(w, extra, offset), out[0], bias=bias,
                        residual=pitched(res, extra + 1, offset), preact=out[1], weight_layout=layout)
    z64, mag = forward64(x, w, layout, bias)
    check_product(out[1], z64, mag, k, 0.0, "z")
    check_product(out[0], z64 + res.double(), mag, k, 2 * U * (z64.abs() + res.double().abs()), "y")
    for o in out:                                             # nothing was written between the rows
        assert torch.isnan(o._base.view(-1)).sum() == offset + m * extra


@pytest.mark.parametrize("layout", [WEIGHT_KN, WEIGHT_NK])
@pytest.mark.parametrize("act", [ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 64, 96), (5, 70, 33), (130, 200, 264), (257, 129, 511), (700, 260, 130)])
def test_backward(h, m, n, k, act, layout):
    x, w = rand(11, m, k), rand(12, *((n, k) if layout == WEIGHT_NK else (k, n)))
    z, dy = rand(13, m, n, scale=3.0), rand(14, m, n, scale=1e-7)     # gradients far below FP16's normal range
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(n, device=DEV)
    h.sgemm_cube_linear_backward(dy, x, w, dX=dx, dW=dw, dbias=db, preact=z, activation=act, weight_layout=layout)
    check_gradients(x, w, z, dy, dx, dw, db, act, layout)


def check_gradients(x, w, z, dy, dx, dw, db, act, layout):
    m, n = dy.shape
    slope = slope64(z.double(), act) if act else torch.ones_like(z, dtype=torch.float64)
    dz, slack = dy.double() * slope, dy.double().abs() * 2.0 ** -20
    wk = w.double() if layout == WEIGHT_NK else w.double().t()        # outputs x inputs
    check_product(dx, dz @ wk, dz.abs() @ wk.abs(), n, slack @ wk.abs(), "dx")
    want, mag, extra = dz.t() @ x.double(), dz.abs().t() @ x.double().abs(), slack.t() @ x.double().abs()
    if layout == WEIGHT_KN:
        want, mag, extra = want.t(), mag.t(), extra.t()
    check_product(dw, want, mag, m, extra, "dw")
    if db is not None:
        err = (db.double() - dz.sum(0)).abs()
        assert bool((err <= (m + 4) * U * dz.abs().sum(0) + slack.sum(0)).all())


@pytest.mark.parametrize("layout", [WEIGHT_KN, WEIGHT_NK])
def test_backward_packed_strided_and_partial(h, layout):
    m, n, k, act = 190, 150, 210, ACT_SILU
    x, w = rand(15, m, k), rand(16, *((n, k) if layout == WEIGHT_NK else (k, n)))
    z, dy = rand(17, m, n), rand(18, m, n)
    xp, wp = PackedMatrix(m, k), PackedMatrix(*w.shape)
    h.sgemm_cube_pack(x, xp)
    h.sgemm_cube_pack(w, wp)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(n, device=DEV)
    h.sgemm_cube_linear_backward(dy, xp, wp, dX=dx, dW=dw, dbias=db, preact=z, activation=act, weight_layout=layout)
    check_gradients(x, w, z, dy, dx, dw, db, act, layout)
    # each gradient by itself, strided, FP32 operands: the same bits
    args = dict(preact=pitched(z, 3, 1), activation=act, weight_layout=layout)
    only = pitched(torch.zeros_like(x), 5, 2)
    h.sgemm_cube_linear_backward(pitched(dy, 1), x, w, dX=only, **args)
    assert torch.equal(only, dx)
    only = pitched(torch.zeros_like(w), 3)
    h.sgemm_cube_linear_backward(pitched(dy, 1), pitched(x, 2), w, dW=only, **args)
    assert torch.equal(only, dw)
    only = torch.zeros(n, device=DEV)
    h.sgemm_cube_linear_backward(dy, x, w, dbias=only, preact=z, activation=act, weight_layout=layout)
    assert torch.equal(only, db)


@pytest.mark.parametrize("m", [3, 200])
def test_gradient_against_differences(h, m):
    """<gradient, v> against the change of the layer's own output along v: truncation e^2/6 |L'''| and FP32 noise
    2^-22 |terms| / e, both under 1e-3 of the gradient's size at e = 2^-6."""
    n, k, e = 96, 64, 2.0 ** -6
    x, w, b, dy = rand(19, m, k), rand(20, k, n, scale=k ** -0.5), rand(21, n), rand(22, m, n)
    y, z = torch.empty(m, n, device=DEV), torch.empty(m, n, device=DEV)
    for act in (ACT_GELU, ACT_GELU_TANH, ACT_SILU):
        h.sgemm_cube_linear(x, w, y, bias=b, activation=act, preact=z)
        grads = [torch.empty_like(t) for t in (x, w, b)]
        h.sgemm_cube_linear_backward(dy, x, w, dX=grads[0], dW=grads[1], dbias=grads[2], preact=z, activation=act)
        for i, t in enumerate((x, w, b)):
            v = torch.sign(grads[i]) / math.sqrt(t.numel())
            values = []
            for s in (e, -e):
                moved = [x, w, b]
                moved[i] = t + s * v
                h.sgemm_cube_linear(moved[0], moved[1], y, bias=moved[2], activation=act)
                values.append((y.double() * dy.double()).sum())
            slope, want = (values[0] - values[1]) / (2 * e), (grads[i].double() * v.double()).sum()
            assert abs(slope - want) <= 2e-3 * want, (act, i, float(slope), float(want))


@pytest.mark.parametrize("sx,sw", [(1e-30, 1e20), (1e30, 1e-25), (2.0 ** -140, 1.0), (1e18, 1e18)])
@pytest.mark.parametrize("m", [2, 140])
def test_magnitudes_of_the_whole_fp32_range(h, m, sx, sw):
    n, k = 130, 192
    x, w = rand(23, m, k, scale=sx), rand(24, n, k, scale=sw)
    y = torch.empty(m, n, device=DEV)
    h.sgemm_cube_linear(x, w, y, weight_layout=WEIGHT_NK)
    z64, mag = forward64(x, w, WEIGHT_NK, None)
    if sx > 2.0 ** -130:
        check_product(y, z64, mag, k, 0.0, "range")
    else:                                                     # FP32 subnormal outputs: absolute spacing 2^-149
        assert float((y.double() - z64).abs().max()) <= 2.0 ** -148 + 2 * k * U * float(mag.max())


def test_wide_spread_inside_an_operand(h):
    """Rows 2^-29 below the largest keep 22 bits; rows further down are off by 2^-51 of the largest at most."""
    m, n, k = 160, 140, 256
    x, w = rand(25, m, k), rand(26, n, k)
    e = torch.arange(m, device=DEV) % 5 * -14.0                # 2^0 .. 2^-56
    x = x * torch.exp2(e)[:, None]
    y = torch.empty(m, n, device=DEV)
    h.sgemm_cube_linear(x, w, y, weight_layout=WEIGHT_NK)
    z64, mag = forward64(x, w, WEIGHT_NK, None)
    floor = 2.0 ** -51 * x.double().abs().max() * w.double().abs().sum(1)
    assert bool(((y.double() - z64).abs() <= 2 * k * U * mag + floor[None, :]).all())
    for step in (0, 1):                                        # within 2^-29 (2^-14 and the rows' own spread)
        rows = (torch.arange(m, device=DEV) % 5) == step
        assert float((y.double() - z64)[rows].norm() / z64[rows].norm()) <= (8 + k / 128) * 2 * U + 2.0 ** -21


def test_nonfinite_entries_stay_in_their_row(h):
    for m in (4, 150):
        x, w = rand(27, m, 96), rand(28, 80, 96)
        want = torch.empty(m, 80, device=DEV)
        h.sgemm_cube_linear(x, w, want, weight_layout=WEIGHT_NK)
        x[1, 5], x[3, 0] = math.inf, math.nan
        y = torch.empty(m, 80, device=DEV)
        h.sgemm_cube_linear(x, w, y, weight_layout=WEIGHT_NK)
        bad = torch.zeros(m, dtype=torch.bool, device=DEV)
        bad[1] = bad[3] = True
        assert not torch.isfinite(y[bad]).any()
        assert torch.isfinite(y[~bad]).all()
        assert float((y - want)[~bad].norm() / want[~bad].norm()) <= 2.0 ** -21


def test_pack_words_and_exponent(h):
    """The words against numpy's FP16 conversions of 2^p x, odd width, zero columns up to the next eighth."""
    for scale in (1.0, 1e-9, 3e7):
        x = rand(29, 37, 61, scale=scale)
        p = PackedMatrix(37, 61)
        p.hi.fill_(7.0)
        p.lo.fill_(7.0)
        h.sgemm_cube_pack(x, p)
        rng = h.sgemm_cube_hi_exponent_range(x)
        e = int(p.exp.item())
        assert e == 15 - rng[1]
        xs = np.ldexp(x.cpu().numpy().astype(np.float64), e)
        hi = xs.astype(np.float16)
        lo = np.ldexp(xs - hi.astype(np.float64), 11).astype(np.float16)
        assert np.array_equal(p.hi[:, :61].cpu().numpy(), hi) and np.array_equal(p.lo[:, :61].cpu().numpy(), lo)
        assert not p.hi[:, 61:].any() and not p.lo[:, 61:].any()
    p = PackedMatrix(3, 8)
    h.sgemm_cube_pack(torch.zeros(3, 8, device=DEV), p)
    assert int(p.exp.item()) == 0 and not p.hi.any() and not p.lo.any()


def test_residual_in_place_and_repeatable(h):
    m, n, k = 300, 260, 2048
    x, w, r = rand(30, m, k), rand(31, n, k), rand(32, m, n)
    y = torch.empty(m, n, device=DEV)
    h.sgemm_cube_linear(x, w, y, residual=r, activation=ACT_GELU, weight_layout=WEIGHT_NK)
    for _ in range(3):
        again = r.clone()
        h.sgemm_cube_linear(x, w, again, residual=again, activation=ACT_GELU, weight_layout=WEIGHT_NK)
        assert torch.equal(again, y)


def test_empty_problems(h):
    b, r = rand(33, 6), rand(34, 4, 6)
    y = torch.full((4, 6), float("nan"), device=DEV)
    h.sgemm_cube_linear(torch.empty(4, 0, device=DEV), torch.empty(0, 6, device=DEV), y, bias=b, residual=r,
                        activation=ACT_RELU)
    assert torch.equal(y, torch.relu(b)[None] + r)
    h.sgemm_cube_linear(torch.empty(0, 5, device=DEV), rand(35, 5, 6), torch.empty(0, 6, device=DEV))
    h.sgemm_cube_linear(rand(35, 4, 5), torch.empty(5, 0, device=DEV), torch.empty(4, 0, device=DEV))
    dw, db = torch.full((5, 6), 1.0, device=DEV), torch.full((6,), 1.0, device=DEV)
    h.sgemm_cube_linear_backward(torch.empty(0, 6, device=DEV), torch.empty(0, 5, device=DEV), rand(35, 5, 6), dW=dw, dbias=db)
    assert not dw.any() and not db.any()
    dx = torch.full((4, 5), 1.0, device=DEV)
    h.sgemm_cube_linear_backward(torch.empty(4, 0, device=DEV), rand(36, 4, 5), torch.empty(5, 0, device=DEV), dX=dx)
    assert not dx.any()


def test_options_give_the_same_layer(h):
    """Pairs, single blocks and split-K realise the same sums (split-K in other brackets)."""
    m, n, k = 400, 300, 1536
    x, w = rand(37, m, k), rand(38, k, n)
    z64, mag = forward64(x, w, WEIGHT_KN, None)
    out = []
    try:
        for pair, split in ((0, 0), (1, 0), (2, 1)):
            h.sgemm_cube_set_option(binding.OPT_CTA_PAIR, pair)
            h.sgemm_cube_set_option(binding.OPT_SPLIT_K, split)
            y = torch.empty(m, n, device=DEV)
            h.sgemm_cube_linear(x, w, y)
            check_product(y, z64, mag, k, 0.0, "pair %d split %d" % (pair, split))
            out.append(y)
    finally:
        h.sgemm_cube_set_option(binding.OPT_CTA_PAIR, 2)
        h.sgemm_cube_set_option(binding.OPT_SPLIT_K, 1)
    assert torch.equal(out[0], out[1])


def test_capture_and_other_stream():
    h = binding.Handle(0)
    try:
        m, n, k = 150, 200, 300
        x, w, b, dy = rand(39, m, k), rand(40, n, k), rand(41, n), rand(42, m, n)
        y, z = torch.empty(m, n, device=DEV), torch.empty(m, n, device=DEV)
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)

        def step(stream=None):
            h.sgemm_cube_linear(x, w, y, bias=b, activation=ACT_GELU, preact=z, weight_layout=WEIGHT_NK, stream=stream)
            h.sgemm_cube_linear_backward(dy, x, w, dX=dx, dW=dw, dbias=db, preact=z, activation=ACT_GELU,
                                         weight_layout=WEIGHT_NK, stream=stream)

        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, dx, dw, db)]
        for t in (y, dx, dw, db):
            t.zero_()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        step(side)
        side.synchronize()
        assert all(torch.equal(a, t) for a, t in zip(want, (y, dx, dw, db)))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        x.mul_(2.0)
        graph.replay()
        torch.cuda.synchronize()
        check_product(z, *forward64(x, w, WEIGHT_NK, b), k, 0.0, "replay")
        assert h.sgemm_cube_check()[0] == 0
    finally:
        h.destroy()


def refused(status, call, *args, **kw):
    with pytest.raises(binding.SgemmCubeError) as e:
        call(*args, **kw)
    assert e.value.status == status


def test_refusals(h):
    x, w, y = rand(43, 4, 8), rand(44, 8, 6), torch.empty(4, 6, device=DEV)
    refused(binding.INVALID_ARG, h.sgemm_cube_linear, x, w, y, activation=5)
    refused(binding.INVALID_ARG, h.sgemm_cube_linear, x, w, y, activation=-1)
    refused(binding.INVALID_ARG, h.sgemm_cube_linear, x, w, y, preact=y)
    refused(binding.INVALID_ARG, h.sgemm_cube_linear_backward, y, x, w, dX=torch.empty_like(x), activation=ACT_GELU)
    with pytest.raises(AssertionError):
        h.sgemm_cube_linear(x, w, torch.empty(4, 5, device=DEV))
    with pytest.raises(AssertionError):
        h.sgemm_cube_linear(x.half(), w, y)
    with pytest.raises(AssertionError):
        h.sgemm_cube_linear(x, w, y, bias=torch.empty(5, device=DEV))
    lib, vp = binding.load(), x.data_ptr()
    good = binding._Operand(vp, 8, None, None, 0, None)
    wo = binding._Operand(w.data_ptr(), 6, None, None, 0, None)

    def call(m=4, n=6, k=8, xo=good, wo=wo, layout=0, ldr=6, r=None, out=y.data_ptr(), ldy=6):
        return lib.sgemm_cube_linear(h._h, m, n, k, xo, wo, layout, None, r, ldr, 0, out, ldy, None, 0, None)

    bad = binding.INVALID_ARG
    assert call(m=-1) == bad and call(layout=2) == bad and call(out=None) == bad and call(ldy=5) == bad
    assert call(r=vp, ldr=5) == bad and call(xo=binding._Operand(vp, 7, None, None, 0, None)) == bad
    assert call(xo=binding._Operand(None, 0, None, None, 0, None)) == bad and call(xo=None) == bad
    p = PackedMatrix(8, 6)
    o = p.operand
    assert call(wo=binding._Operand(None, 0, o.hi_dev, o.lo_dev, o.ld16, None)) == bad
    assert call(wo=binding._Operand(None, 0, o.hi_dev + 2, o.lo_dev, o.ld16, o.exp_dev)) == binding.MISALIGNED
    assert call(wo=binding._Operand(None, 0, o.hi_dev, o.lo_dev, 6, o.exp_dev)) == binding.MISALIGNED
    assert lib.sgemm_cube_pack(h._h, 8, 6, w.data_ptr(), 6, o.hi_dev, o.lo_dev, 6, o.exp_dev, None) == binding.MISALIGNED
    assert lib.sgemm_cube_pack(h._h, 8, 6, w.data_ptr(), 5, o.hi_dev, o.lo_dev, 8, o.exp_dev, None) == bad
    assert lib.sgemm_cube_pack(h._h, 8, 6, None, 6, o.hi_dev, o.lo_dev, 8, o.exp_dev, None) == bad
    assert lib.sgemm_cube_linear(None, 4, 6, 8, good, wo, 0, None, None, 0, 0, y.data_ptr(), 6, None, 0, None) == bad
