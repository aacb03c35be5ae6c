"""Linear layers of short batches: the weight on the wide side of the tile, X (and an FP32 weight) split block by block
of 64 inputs, each block with an exponent of its own.  Sizes on both sides of every limit of the choice of kernel.

Tolerance: the product's (componentwise max(2 K, K + 14) u |x||w| and (8 + K / 128) 2^-23 + 2^-21 in the Frobenius norm,
u = 2^-24); the blocks' sums meet in FP32, one rounding per 64 inputs, which the first covers."""
import math

import pytest
import torch

from paper_2507_23387_b200 import binding
from paper_2507_23387_b200.binding import (ACT_GELU, ACT_GELU_TANH, ACT_NONE, ACT_RELU, ACT_SILU, WEIGHT_KN, WEIGHT_NK,
                                           PackedMatrix)

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


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


def weight(seed, n, k, layout):
    return rand(seed, *((n, k) if layout == WEIGHT_NK else (k, n)))


def close(got, x, w, layout, bias=None, frob=True):
    wk = w.double().t() if layout == WEIGHT_NK else w.double()
    want, mag = x.double() @ wk, x.double().abs() @ wk.abs()
    if bias is not None:
        want, mag = want + bias.double(), mag + bias.double().abs()
    k = x.shape[1]
    err = (got.double() - want).abs()
    assert torch.isfinite(got).all()
    assert bool((err <= max(2 * k, k + 14) * U * 1.2 * mag).all()), float((err / mag).max())
    if frob:
        assert float(err.norm() / want.norm()) <= (8 + k / 128) * 2 * U + 2.0 ** -21


def both_weights(h, w):
    p = PackedMatrix(*w.shape)
    h.sgemm_cube_pack(w, p)
    return (("words", p), ("fp32", w))


@pytest.mark.parametrize("layout", [WEIGHT_KN, WEIGHT_NK])
@pytest.mark.parametrize("n,k", [(1, 1), (5, 64), (127, 65), (128, 63), (129, 128), (300, 520), (1000, 1027), (260, 4100)])
@pytest.mark.parametrize("m", [2, 4, 5, 8, 9, 16, 17, 32, 33, 64, 65, 128, 129, 200, 256, 257])
def test_sizes(h, m, n, k, layout):
    x, w, b = rand(m, m, k), weight(1000 + n, n, k, layout), rand(3, n)
    for _, op in both_weights(h, w):
        y = torch.full((m, n), float("nan"), device=DEV)
        h.sgemm_cube_linear(x, op, y, bias=b, weight_layout=layout)
        close(y, x, w, layout, b)


@pytest.mark.parametrize("layout", [WEIGHT_KN, WEIGHT_NK])
@pytest.mark.parametrize("m,n,k", [(24, 16500, 200), (64, 19000, 130), (100, 5000, 700), (160, 3000, 2100)])
def test_more_tiles_than_processors_and_turns(h, m, n, k, layout):
    x, w = rand(4, m, k), weight(5, n, k, layout)
    for _, op in both_weights(h, w):
        y = torch.full((m, n), float("nan"), device=DEV)
        h.sgemm_cube_linear(x, op, y, weight_layout=layout)
        close(y, x, w, layout)


@pytest.mark.parametrize("act", [ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU])
@pytest.mark.parametrize("m,n,k", [(20, 200, 330), (50, 140, 2048), (130, 150, 700)])
def test_epilogue(h, m, n, k, act):
    f = {ACT_NONE: lambda z: z, ACT_RELU: torch.relu, ACT_GELU: torch.nn.functional.gelu, ACT_SILU: torch.nn.functional.silu,
         ACT_GELU_TANH: lambda z: torch.nn.functional.gelu(z, approximate="tanh")}[act]
    x, w, b, r = rand(6, m, k), rand(7, n, k, scale=k ** -0.5), rand(8, n), rand(9, m, n)
    for _, op in both_weights(h, w):
        y, z = r.clone(), torch.full((m, n), float("nan"), device=DEV)
        h.sgemm_cube_linear(x, op, y, bias=b, residual=y, activation=act, preact=z, weight_layout=WEIGHT_NK)
        close(z, x, w, WEIGHT_NK, b)
        want = f(z.double()) + r.double()
        assert bool(((y.double() - want).abs() <= 2.0 ** -21 * (1 + z.double().abs()) + 2 * U * want.abs()).all())
        again = torch.empty_like(y)
        h.sgemm_cube_linear(x, op, again, bias=b, residual=r, activation=act, weight_layout=WEIGHT_NK)
        assert torch.equal(again, y)


@pytest.mark.parametrize("extra,offset", [(1, 0), (4, 0), (4, 1), (3, 2)])
@pytest.mark.parametrize("layout", [WEIGHT_KN, WEIGHT_NK])
def test_strides_and_alignment(h, layout, extra, offset):
    def pitched(t):
        r, c = t.shape
        buf = torch.full((r * (c + extra) + offset,), float("nan"), device=DEV)
        v = buf[offset:offset + r * (c + extra)].view(r, c + extra)[:, :c]
        return v.copy_(t)

    m, n, k = 40, 136, 200
    x, w, r = rand(10, m, k), weight(11, n, k, layout), rand(12, m, n)
    for name, op in both_weights(h, pitched(w)):
        y, z = pitched(torch.zeros(m, n, device=DEV)), pitched(torch.zeros(m, n, device=DEV))
        before = y.storage()
        guard = torch.tensor(before.tolist(), device=DEV)
        h.sgemm_cube_linear(pitched(x), op, y, residual=pitched(r), preact=z, weight_layout=layout)
        close(z, x, w, layout)
        assert bool(((y.double() - z.double() - r.double()).abs() <= U * y.double().abs()).all())
        after = torch.tensor(before.tolist(), device=DEV)           # nothing between the rows was written
        outside = torch.isnan(guard)
        assert torch.isnan(after[outside]).all() and torch.isfinite(after[~outside]).all()


@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("step", [7, 40, 120])
def test_blocks_of_very_different_size(h, order, step):
    """Blocks of 64 inputs that grow or shrink by 2^step from one to the next, zero blocks between them; a row that lives
    in the smallest block alone keeps its precision while FP32 holds it."""
    m, n, blocks = 24, 140, 7
    k = 64 * blocks
    if step * (blocks - 1) > 120:
        blocks = 120 // step + 1
    e = (torch.arange(k, device=DEV) // 64).clamp(max=blocks - 1) * float(step) - 60.0
    if order < 0:
        e = e.flip(0)
    x = rand(13, m, k) * torch.exp2(e)[None]
    small = e == e.min()
    x[5] = torch.where(small, x[5], torch.zeros_like(x[5]))
    x[:, 128:192] = 0.0
    x[7] = 0.0
    for layout in (WEIGHT_NK, WEIGHT_KN):
        w = weight(14, n, k, layout)
        for _, op in both_weights(h, w):
            y = torch.empty(m, n, device=DEV)
            h.sgemm_cube_linear(x, op, y, weight_layout=layout)
            wk = w.double().t() if layout == WEIGHT_NK else w.double()
            live = torch.ones(m, dtype=torch.bool, device=DEV)
            live[7] = False
            assert not y[7].any()
            if step < 40:                                  # the words of a small block of FP32 weights and rows: all bits
                close(y[live], x[live], w, layout, frob=False)
            else:
                keep = live.clone()
                keep[5] = False
                close(y[keep], x[keep], w, layout, frob=False)
                want, mag = x[5].double() @ wk, x[5].double().abs() @ wk.abs()
                assert bool(((y[5].double() - want).abs() <= 2 * k * U * 1.2 * mag + 2.0 ** -148).all())


@pytest.mark.parametrize("sx,sw", [(1e-30, 1e20), (1e30, 1e-25), (2.0 ** -140, 1.0), (1e18, 1e18), (1e-25, 1e-10)])
@pytest.mark.parametrize("m", [12, 60])
def test_magnitudes(h, m, sx, sw):
    n, k = 130, 1192
    x, w = rand(15, m, k, scale=sx), rand(16, n, k, scale=sw)
    for _, op in both_weights(h, w):
        y = torch.empty(m, n, device=DEV)
        h.sgemm_cube_linear(x, op, y, weight_layout=WEIGHT_NK)
        if sx > 2.0 ** -130:
            close(y, x, w, WEIGHT_NK)
        else:                                              # FP32 subnormal results: absolute spacing 2^-149
            mag = x.double().abs() @ w.double().abs().t()
            assert float((y.double() - x.double() @ w.double().t()).abs().max()) <= 2.0 ** -148 + 2 * k * U * float(mag.max())


def test_nonfinite_entries_stay_in_their_row_and_column(h):
    m, n, k = 30, 150, 400
    x, w = rand(17, m, k), rand(18, n, k)
    x[1, 5], x[3, 350], x[4, 2] = math.inf, math.nan, -math.inf
    w[7, 9], w[140, 399] = math.nan, math.inf
    bad = torch.zeros(m, n, dtype=torch.bool, device=DEV)
    bad[[1, 3, 4]] = True
    bad[:, [7, 140]] = True
    clean_x, clean_w = torch.where(torch.isfinite(x), x, 0.0 * x.new_ones(())), torch.where(torch.isfinite(w), w, 0.0 * w.new_ones(()))
    want, mag = clean_x.double() @ clean_w.double().t(), clean_x.double().abs() @ clean_w.double().abs().t()
    for _, op in both_weights(h, w):
        y = torch.empty(m, n, device=DEV)
        h.sgemm_cube_linear(x, op, y, weight_layout=WEIGHT_NK)
        assert not torch.isfinite(y[bad]).any()
        assert torch.isfinite(y[~bad]).all()
        assert bool(((y.double() - want).abs()[~bad] <= (2 * k * U * 1.2 * mag)[~bad]).all())


def test_repeatable_streams_capture_and_without_split_k():
    h = binding.Handle(0)
    try:
        for m, n, k in ((24, 500, 3000), (100, 300, 900)):
            x, w = rand(19, m, k), rand(20, n, k)
            for _, op in both_weights(h, w):
                y = torch.empty(m, n, device=DEV)

                def call(stream=None):
                    h.sgemm_cube_linear(x, op, y, weight_layout=WEIGHT_NK, stream=stream)

                call()
                want = y.clone()
                torch.cuda.synchronize()
                side = torch.cuda.Stream()
                y.zero_()
                torch.cuda.synchronize()
                call(side)
                side.synchronize()
                assert torch.equal(y, want)
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    call()
                y.zero_()
                graph.replay()
                assert torch.equal(y, want)
                h.sgemm_cube_set_option(binding.OPT_SPLIT_K, 0)
                call()
                close(y, x, w, WEIGHT_NK)
                h.sgemm_cube_set_option(binding.OPT_SPLIT_K, 1)
        assert h.sgemm_cube_check()[0] == 0
    finally:
        h.destroy()
