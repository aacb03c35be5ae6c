"""The language-model operators where sizes, strides and callers reach further than usual: operands packed in more than
one launch, several waves of tiles, offsets past 2^31 elements, streams, captured graphs, ends of the scale's range."""
import pytest
import torch

from paper_2507_23387_b200 import binding
from paper_2507_23387_b200.binding import ACT_SILU, WEIGHT_KN, WEIGHT_NK, PackedMatrix

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    torch.cuda.synchronize()
    handle.destroy()


def rand(seed, *shape, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV) * scale


def close(got, a, b, plus=None):
    """got = a b + plus: componentwise 2 K u |a||b|, and (8 + K / 128) 2^-23 + 2^-21 in the Frobenius norm."""
    want, mag = a.double() @ b.double(), a.double().abs() @ b.double().abs()
    if plus is not None:
        want, mag = want + plus.double(), mag + plus.double().abs()
    k = a.shape[1]
    err = (got.double() - want).abs()
    assert torch.isfinite(got).all()
    assert bool((err <= max(2 * k, k + 14) * U * 1.2 * mag).all())
    assert float(err.norm() / want.norm()) <= (8 + k / 128) * 2 * U + 2.0 ** -21


# operands past what one cooperative packing launch holds; sizes on both sides of multiples of 8 and of tiles
@pytest.mark.parametrize("m,n,k,layout", [(2304, 2000, 2500, WEIGHT_KN), (2303, 2001, 2501, WEIGHT_NK), (2305, 1999, 2503, WEIGHT_KN)])
def test_large_operands_forward_and_backward(h, m, n, k, layout):
    x, w, r, dy = rand(1, m, k), rand(2, *((k, n) if layout == WEIGHT_KN else (n, k))), rand(3, m, n), rand(4, m, n, scale=1e-4)
    wkn = w if layout == WEIGHT_KN else w.t()
    y, dx, dw, db = torch.empty_like(r), torch.empty_like(x), torch.empty_like(w), torch.empty(n, device=DEV)
    h.sgemm_cube_linear(x, w, y, residual=r, weight_layout=layout)
    close(y, x, wkn, r)
    h.sgemm_cube_linear_backward(dy, x, w, dX=dx, dW=dw, dbias=db, weight_layout=layout)
    close(dx, dy, wkn.t())
    close(dw if layout == WEIGHT_KN else dw.t(), x.t(), dy)
    want = dy.double().sum(0)
    assert bool(((db.double() - want).abs() <= m * U * dy.double().abs().sum(0)).all())
    # the gradient through an activation, of the same operands
    z = rand(5, m, n)
    h.sgemm_cube_linear_backward(dy, x, w, dX=dx, dbias=db, preact=z, activation=ACT_SILU, weight_layout=layout)
    s = torch.sigmoid(z.double())
    d = dy.double() * s * (1 + z.double() * (1 - s))
    err = (dx.double() - d @ wkn.double().t()).abs()
    mag = d.abs() @ wkn.double().abs().t()
    # the activation's slope in FP32 adds at most 2^-20 of each of dy's entries
    assert bool((err <= (2 * n * U * 1.2 + 2.0 ** -20) * mag + 2.0 ** -20 * (dy.double().abs() @ wkn.double().abs().t())).all())
    assert h.sgemm_cube_check()[0] == 0


def far(rows, cols, ld, dtype=torch.float32):
    buf = torch.empty((rows - 1) * ld + cols, dtype=dtype, device=DEV)
    return torch.as_strided(buf, (rows, cols), (ld, 1))


@pytest.mark.parametrize("m", [5, 9])
@pytest.mark.parametrize("layout", [WEIGHT_KN, WEIGHT_NK])
def test_linear_offsets_past_32_bits(h, m, layout):
    """One matrix after the other with rows that lie 2^29 elements and more apart."""
    n, k, ld = 24, 12, 540_000_001 if m == 5 else 300_000_000
    x, r, dy = rand(6, m, k), rand(7, m, n), rand(8, m, n)
    w = rand(9, *((k, n) if layout == WEIGHT_KN else (n, k)))
    wkn = w if layout == WEIGHT_KN else w.t()
    y, dx = torch.empty(m, n, device=DEV), torch.empty(m, k, device=DEV)
    fx = far(m, k, ld).copy_(x)
    h.sgemm_cube_linear(fx, w, y, residual=r, weight_layout=layout)
    close(y, x, wkn, r)
    h.sgemm_cube_linear_backward(dy, x, w, dX=fx, weight_layout=layout)
    close(fx.contiguous(), dy, wkn.t())
    del fx
    fy = far(m, n, ld).copy_(r)
    h.sgemm_cube_linear(x, w, fy, residual=fy, weight_layout=layout)
    close(fy.contiguous(), x, wkn, r)
    fy.copy_(dy)
    h.sgemm_cube_linear_backward(fy, x, w, dX=dx, weight_layout=layout)
    close(dx, dy, wkn.t())
    del fy
    rows = w.shape[0]
    fw = far(rows, w.shape[1], 2 ** 31 // (rows - 1) + 1).copy_(w)
    h.sgemm_cube_linear(x, fw, y, weight_layout=layout)
    close(y, x, wkn)
    p = PackedMatrix(*w.shape)
    h.sgemm_cube_pack(fw, p)
    h.sgemm_cube_linear(x, p, y, weight_layout=layout)
    close(y, x, wkn)
    h.sgemm_cube_linear_backward(dy, x, w, dW=fw, weight_layout=layout)
    dw = fw.contiguous() if layout == WEIGHT_KN else fw.contiguous().t()
    close(dw, x.t(), dy)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_offsets_past_32_bits(h, dtype):
    rows, cols, ld = 5, 1000, 540_000_000
    x, w, dy = rand(10, rows, cols).to(dtype), rand(11, cols), rand(12, rows, cols).to(dtype)
    mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    h.sgemm_cube_layer_norm(x, y, w, None, mean=mean, rstd=rstd)
    h.sgemm_cube_layer_norm_backward(dy, x, mean, rstd, dx, w)
    f = far(rows, cols, ld, dtype).copy_(x)
    h.sgemm_cube_layer_norm(f, f, w, None)
    assert torch.equal(f.contiguous(), y)
    f.copy_(dy)
    h.sgemm_cube_layer_norm_backward(f, x, mean, rstd, f, w)
    assert torch.equal(f.contiguous(), dx)


def test_norm_and_logprobs_on_another_stream_and_captured():
    h = binding.Handle(0)
    try:
        rows, cols, k = 70, 1003, 6
        x, w, dy = rand(13, rows, cols), rand(14, cols), rand(15, rows, cols)
        t = torch.arange(rows, device=DEV) * 11 % cols
        y, dx, g = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
        dw, db, mean, rstd, lp, en = [torch.empty(n, device=DEV) for n in (cols, cols, rows, rows, rows, rows)]
        st, tl, ti = torch.empty(rows, 2, device=DEV), torch.empty(rows, k, device=DEV), torch.empty(rows, k, dtype=torch.int64, device=DEV)
        out = [y, dx, dw, db, mean, rstd, lp, en, st, tl, ti, g]

        def step(stream=None):
            h.sgemm_cube_layer_norm(x, y, w, None, mean=mean, rstd=rstd, stream=stream)
            h.sgemm_cube_layer_norm_backward(dy, x, mean, rstd, dx, w, dw, db, stream=stream)
            h.sgemm_cube_token_logprobs(y, t, lp, entropy=en, stats=st, top_logp=tl, top_index=ti, stream=stream)
            h.sgemm_cube_token_logprobs_backward(y, t, st, g, dlogp=mean, entropy=en, dentropy=rstd, stream=stream)

        def again(run):
            for o in out:
                o.zero_()
            torch.cuda.synchronize()
            run()
            torch.cuda.synchronize()
            return [o.clone() for o in out]

        want = again(step)
        assert all(torch.isfinite(o.double()).all() for o in want)
        side = torch.cuda.Stream()
        assert all(torch.equal(a, b) for a, b in zip(want, again(lambda: step(side))))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        assert all(torch.equal(a, b) for a, b in zip(want, again(graph.replay)))
        x.mul_(-3.0)
        moved = again(graph.replay)
        assert all(torch.equal(a, b) for a, b in zip(moved, again(step)))
        assert not torch.equal(moved[0], want[0])
        assert h.sgemm_cube_check()[0] == 0
    finally:
        h.destroy()


def test_ends_of_the_scale(h):
    """scale = 2^-30: all probabilities equal; 2^30: the largest logit takes all, at distances of 1 and more."""
    rows, vocab = 3, 777
    x = (torch.arange(rows * vocab, device=DEV).view(rows, vocab) * 31 % vocab).float()
    t = x.argmax(1)
    lp, en = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    h.sgemm_cube_token_logprobs(x, t, lp, entropy=en, scale=2.0 ** 30)
    assert bool((lp == 0).all()) and bool((en == 0).all())
    h.sgemm_cube_token_logprobs(x, t, lp, entropy=en, scale=2.0 ** -30)
    ln = torch.tensor(float(vocab), dtype=torch.float64).log()
    assert bool(((lp.double() + ln).abs() <= 1e-5).all()) and bool(((en.double() - ln).abs() <= 1e-5).all())
    for scale in (2.0 ** 31, 1.5 * 2.0 ** 30, 2.0 ** -31, 1e-38, -2.0 ** 5):
        with pytest.raises(binding.SgemmCubeError) as err:
            h.sgemm_cube_token_logprobs(x, t, lp, scale=scale)
        assert err.value.status == binding.INVALID_ARG
        with pytest.raises(binding.SgemmCubeError) as err:
            h.sgemm_cube_token_logprobs_backward(x, t, torch.empty(rows, 2, device=DEV), torch.empty_like(x), dlogp=lp, scale=scale)
        assert err.value.status == binding.INVALID_ARG


@pytest.mark.parametrize("scale", [3e4, 1e7, 2.0 ** 28])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_large_scaled_logits(h, scale, dtype):
    """Scaled logits far past what FP32 resolves to a unit: the distances to the largest one still decide."""
    rows, vocab = 5, 9001
    g = torch.Generator(device=DEV).manual_seed(21)
    x = torch.randn((rows, vocab), generator=g, device=DEV).mul_(3).to(dtype)
    x[3] += 40000.0                                       # many equal ones in a row
    x[4] -= 3e4
    t = torch.stack([x[r].float().topk(4).indices[r % 4] for r in range(rows)])
    lp, en, st = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV)
    gr, dlp = torch.empty_like(x), torch.randn(rows, generator=g, device=DEV)
    h.sgemm_cube_token_logprobs(x, t, lp, entropy=en, stats=st, scale=scale)
    h.sgemm_cube_token_logprobs_backward(x, t, st, gr, dlogp=dlp, scale=scale)
    s = torch.tensor(scale, dtype=torch.float32).double().item()
    want = torch.log_softmax(x.double() * s, 1)
    p = want.exp()
    at = want.gather(1, t[:, None])[:, 0]
    ent = -(p * want.clamp(min=-1e300)).sum(1)
    # (x - m) scale is a difference and a product: 2^-23 of itself; base 2 and exp2 add 2^-21 of a term that counts
    assert bool(((lp.double() - at).abs() <= 2.0 ** -21 * (1 + at.abs())).all())
    assert bool(((en.double() - ent).abs() <= 2.0 ** -17 * (1 + ent)).all())
    hot = torch.zeros_like(want).scatter_(1, t[:, None], 1.0)
    wg = s * dlp.double()[:, None] * (hot - p)
    unit = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
    # beyond FP16's range the gradient is infinite on both sides
    fits = wg.abs() < torch.finfo(dtype).max
    err = (gr.double() - wg).abs()
    assert bool((err <= 2.0 ** -17 * s * dlp.abs().double()[:, None] * (hot + p) + unit * wg.abs() + 2.0 ** -25)[fits].all())
