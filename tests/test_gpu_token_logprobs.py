"""Log probabilities of tokens, entropy, top alternatives and the logits' gradient against the definition in FP64.

Tolerances (u = 2^-24).  A term of the sum of exponentials is good to 2^-21 (the instruction's 2^-22, the rounding of
its argument weighted by the term), the sum adds at most depth = 64 + vocab / 512 numbers one after the other; log
probabilities add the rounding of scale (x - m).  The order of the alternatives is exact."""
import math

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


def logits_of(seed, rows, vocab, dtype, scale=3.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn((rows, vocab), generator=g, device=DEV) * scale).to(dtype)


def tokens_of(seed, rows, vocab):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(0, vocab, (rows,), generator=g, device=DEV)


def run(h, x, tokens, top=0, scale=1.0):
    rows = x.shape[0]
    out = {k: torch.full((rows,), 7.0, device=DEV) for k in ("logp", "entropy")}
    out["stats"] = torch.full((rows, 2), 7.0, device=DEV)
    if top:
        out["top_logp"] = torch.full((rows, top), 7.0, device=DEV)
        out["top_index"] = torch.full((rows, top), -7, dtype=torch.int64, device=DEV)
    h.sgemm_cube_token_logprobs(x, tokens, out["logp"], entropy=out["entropy"], stats=out["stats"],
                                top_logp=out.get("top_logp"), top_index=out.get("top_index"), scale=scale)
    return out


def reference(x, tokens, scale=1.0):
    shifted = (x.double() - x.double().amax(1, keepdim=True)) * scale
    logz = torch.logsumexp(shifted, 1)
    logq = shifted - logz[:, None]
    entropy = torch.special.entr(logq.exp()).sum(1)
    t = tokens.clamp(min=0)
    logp = torch.where(tokens >= 0, logq.gather(1, t[:, None])[:, 0], 0.0)
    return logq, logp, entropy, logz


def order(x, k):
    """Columns by value, then by column (a stable sort of the exact values)."""
    return torch.sort(x.float() + 0.0, dim=1, descending=True, stable=True).indices[:, :k]


def check(x, tokens, out, top=0, scale=1.0):
    vocab = x.shape[1]
    logq, logp, entropy, logz = reference(x, tokens, scale)
    rel = 2.0 ** -21 + (64 + vocab / 512) * U
    m = x.double().amax(1)
    def near(got, want, tol):
        same = torch.isfinite(want)
        assert torch.equal(got[~same].double(), want[~same])
        assert bool(((got.double() - want).abs()[same] <= tol.expand_as(want)[same]).all()), float((got.double() - want).abs()[same].max())
    e_logz = rel + 4 * U * logz.abs()
    near(out["logp"], logp, e_logz + 4 * U * (logp.abs() + logz))
    near(out["entropy"], entropy, e_logz + (2 * rel + 4 * U) * (1 + logz + entropy))
    assert torch.equal(out["stats"][:, 0].double(), m)
    assert bool(((out["stats"][:, 1].log().double() - logz).abs() <= e_logz).all())
    if top:
        idx = order(x, top)
        assert torch.equal(out["top_index"], idx)
        want = logq.gather(1, idx)
        near(out["top_logp"], want, (e_logz + 4 * U * logz)[:, None] + 4 * U * want.abs())


# one column; less than a vector; around a vector, a warp, a block's threads; several batches; clusters
VOCABS = [1, 2, 3, 7, 8, 9, 31, 100, 511, 513, 4097, 8192, 8200, 16390, 40003, 131072]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_forward(h, vocab, dtype):
    for rows in (1, 4, 33, 300 if vocab <= 16390 else 5):
        x, t = logits_of(vocab, rows, vocab, dtype), tokens_of(rows, rows, vocab)
        for top in (0, min(vocab, 32), min(vocab, 5)):
            check(x, t, run(h, x, t, top), top)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("extra,offset", [(0, 1), (1, 0), (3, 2), (8, 0)])
def test_strides_and_alignment(h, dtype, extra, offset):
    for rows, vocab in ((6, 5), (7, 1001), (3, 20011), (40, 8192)):
        x, t = logits_of(1, rows, vocab, dtype), tokens_of(2, rows, vocab)
        buf = torch.full((rows * (vocab + extra) + offset,), 1e4, device=DEV).to(dtype)     # neighbours that would win
        v = buf[offset:offset + rows * (vocab + extra)].view(rows, vocab + extra)[:, :vocab]
        v.copy_(x)
        top = min(vocab, 20)
        check(x, t, run(h, v, t, top), top)


@pytest.mark.parametrize("dtype", TYPES)
def test_ties_order_by_column(h, dtype):
    for rows, vocab in ((3, 64), (2, 5000), (2, 70001)):
        x = torch.zeros(rows, vocab, device=DEV, dtype=dtype)                    # all equal
        x[1] = torch.randint(0, 3, (vocab,), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).to(dtype)
        x[0, ::2] = -0.0                                                        # equal to +0
        t = tokens_of(4, rows, vocab)
        for top in (1, 32):
            check(x, t, run(h, x, t, top), top)


@pytest.mark.parametrize("dtype", TYPES)
def test_large_values_in_one_place(h, dtype):
    """The alternatives sit in one thread's columns, in one block's, at the ends, in rising and falling rows."""
    vocab = 65536
    v = 4 if dtype == torch.float32 else 8
    ramp = torch.arange(vocab, device=DEV).float() / vocab
    rows = [ramp, -ramp, -ramp, -ramp, -ramp]
    rows = torch.stack(rows).clone()
    cols = torch.arange(vocab, device=DEV)
    rows[2][(cols // v) % 512 == 77] += 5.0                                     # one thread of every block
    rows[3][(cols // v) % 512 < 3] += 5.0                                       # more than the list of candidates holds
    rows[4][-50:] += 5.0
    x, t = rows.to(dtype), tokens_of(5, 5, vocab)
    for top in (1, 20, 32):
        check(x, t, run(h, x, t, top), top)
    many = x.repeat(70, 1)                                                      # one block a row
    tm = tokens_of(6, 350, vocab)
    check(many, tm, run(h, many, tm, 32), 32)


@pytest.mark.parametrize("dtype", TYPES)
def test_masked_and_empty_rows(h, dtype):
    lowest = torch.finfo(dtype).min
    for vocab in (40, 3001, 33000):
        x = logits_of(7, 7, vocab, dtype)
        t = tokens_of(8, 7, vocab)
        x[0, vocab // 3:] = -math.inf
        x[1] = -math.inf                                       # nothing left
        x[2] = lowest                                          # all lowest: a uniform distribution
        x[3, :-1] = lowest                                     # one left, at the end
        x[4, 1:] = -math.inf                                   # one left, at the front
        x[5] = -math.inf
        x[5, vocab - 2] = lowest                               # the lowest value beats -inf
        t[0], t[4] = vocab - 1, 0                              # a token that is masked, the one that is left
        t[6] = -100
        top = 8
        out = run(h, x, t, top)
        keep = [0, 2, 3, 4, 5, 6]
        check(x[keep], t[keep], {k: o[keep] for k, o in out.items()}, top)
        assert out["logp"][1] == -math.inf and out["entropy"][1] == 0
        assert torch.equal(out["stats"][1], torch.tensor([-math.inf, 0.0], device=DEV))
        assert bool((out["top_logp"][1] == -math.inf).all()) and out["top_index"][1].tolist() == list(range(top))
        assert out["logp"][6] == 0
        d = torch.full_like(x, 7.0)
        g = torch.ones(7, device=DEV)
        h.sgemm_cube_token_logprobs_backward(x, t, out["stats"], d, dlogp=g, entropy=out["entropy"], dentropy=g)
        assert not d[1].any() and torch.isfinite(d).all()
        check_grad(x[keep], t[keep], d[keep], g[keep], g[keep])


def test_nonfinite_rows_stay_apart(h):
    vocab = 20000
    x, t = logits_of(9, 5, vocab, torch.float32), tokens_of(10, 5, vocab)
    x[1, 4], x[3, 11111] = math.nan, math.inf
    t[4] = vocab                                               # out of range
    out = run(h, x, t, 4)
    keep = [0, 2]
    check(x[keep], t[keep], {k: o[keep] for k, o in out.items()}, 4)
    for r in (1, 3):
        assert math.isnan(out["logp"][r]) and math.isnan(out["entropy"][r])
        assert bool(((out["top_index"][r] >= 0) & (out["top_index"][r] < vocab)).all())
    assert math.isnan(out["logp"][4]) and math.isfinite(out["entropy"][4])


@pytest.mark.parametrize("scale", [0.25, 1.0, 7.5, 1000.0])
def test_scale(h, scale):
    x, t = logits_of(11, 9, 6000, torch.float32), tokens_of(12, 9, 6000)
    out = run(h, x, t, 10, scale)
    check(x, t, out, 10, scale)
    g = torch.randn(9, device=DEV)
    d = torch.empty_like(x)
    h.sgemm_cube_token_logprobs_backward(x, t, out["stats"], d, dlogp=g, entropy=out["entropy"], dentropy=g, scale=scale)
    check_grad(x, t, d, g, g, scale)


def check_grad(x, tokens, d, g, hh, scale=1.0):
    vocab = x.shape[1]
    logq, _, entropy, logz = reference(x, tokens, scale)
    p = logq.exp()
    gv = torch.where(tokens >= 0, g.double(), 0.0)[:, None] if g is not None else torch.zeros_like(logz)[:, None]
    hv = hh.double()[:, None] if hh is not None else torch.zeros_like(gv)
    plogq = -torch.special.entr(p)
    want = -p * gv - hv * (plogq + p * entropy[:, None])
    rows = torch.arange(len(tokens), device=DEV)
    want[rows, tokens.clamp(min=0)] += gv[:, 0]
    want = want * scale
    # p is good to rel (statistics and exponential), its argument's rounding 2u|t|; the brackets to their own size
    rel = 2.0 ** -20 + (96 + vocab / 512) * U
    logs = torch.where(p > 0, logq.abs(), 0.0)
    size = p * (gv.abs() + hv.abs() * (logs + entropy[:, None] + 1 + logz[:, None]))
    tol = scale * (3 * rel + 8 * U * logs) * size + (4 * U + ROUND[x.dtype]) * want.abs()
    tol[rows, tokens.clamp(min=0)] += scale * 2 * U * gv[:, 0].abs()
    tol = tol + {torch.float32: 1e-37, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-37}[x.dtype]
    assert torch.isfinite(d).all()
    assert bool(((d.double() - want).abs() <= tol).all()), float(((d.double() - want).abs() - tol).max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 5), (4, 64), (5, 1000), (9, 4099), (200, 2048), (3, 40000), (2, 50001)])
def test_backward(h, rows, vocab, dtype):
    x, t = logits_of(13, rows, vocab, dtype), tokens_of(14, rows, vocab)
    if rows > 2:
        t[1] = -1
    g, e = torch.randn(rows, device=DEV), torch.randn(rows, device=DEV)
    out = run(h, x, t)
    for gg, ee in ((g, e), (g, None), (None, e)):
        d = torch.full_like(x, 7.0)
        h.sgemm_cube_token_logprobs_backward(x, t, out["stats"], d, dlogp=gg, entropy=out["entropy"] if ee is not None else None, dentropy=ee)
        check_grad(x, t, d, gg, ee)
    full = torch.empty_like(x)
    h.sgemm_cube_token_logprobs_backward(x, t, out["stats"], full, dlogp=g, entropy=out["entropy"], dentropy=e)
    inplace = x.clone()
    h.sgemm_cube_token_logprobs_backward(inplace, t, out["stats"], inplace, dlogp=g, entropy=out["entropy"], dentropy=e)
    assert torch.equal(inplace, full)
    for extra, offset in ((1, 0), (8, 0), (0, 1)):
        buf = torch.full((rows * (vocab + extra) + offset,), float("nan"), device=DEV, dtype=dtype)
        v = buf[offset:offset + rows * (vocab + extra)].view(rows, vocab + extra)[:, :vocab]
        h.sgemm_cube_token_logprobs_backward(x, t, out["stats"], v, dlogp=g, entropy=out["entropy"], dentropy=e)
        assert torch.equal(v, full) and torch.isnan(buf).sum() == offset + rows * extra


def test_gradient_against_differences(h):
    rows, vocab, e = 6, 300, 2.0 ** -5
    x, t = logits_of(15, rows, vocab, torch.float32, 1.5), tokens_of(16, rows, vocab)
    g, c = torch.randn(rows, device=DEV), torch.randn(rows, device=DEV)
    out = run(h, x, t)
    d = torch.empty_like(x)
    h.sgemm_cube_token_logprobs_backward(x, t, out["stats"], d, dlogp=g, entropy=out["entropy"], dentropy=c)
    v = torch.sign(d) / x.numel() ** 0.5
    values = []
    for s in (e, -e):
        o = run(h, x + s * v, t)
        values.append((o["logp"].double() * g.double() + o["entropy"].double() * c.double()).sum())
    slope, want = (values[0] - values[1]) / (2 * e), (d.double() * v.double()).sum()
    assert abs(slope - want) <= 2e-3 * want, (float(slope), float(want))


def test_offsets_past_32_bits(h):
    """A leading dimension that puts later rows past 2^31 elements."""
    rows, vocab, ld = 5, 1000, 600_000_000
    buf = torch.empty(4 * ld + vocab, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(buf, (rows, vocab), (ld, 1))
    x.copy_(logits_of(17, rows, vocab, torch.bfloat16))
    t = tokens_of(18, rows, vocab)
    c = x.contiguous()
    out = run(h, x, t, 5)
    check(c, t, out, 5)
    g = torch.randn(rows, device=DEV)
    h.sgemm_cube_token_logprobs_backward(x, t, out["stats"], x, dlogp=g)
    check_grad(c, t, x.contiguous(), g, None)


def test_empty_and_refusals(h):
    e = torch.empty(0, 16, device=DEV)
    v, t0 = torch.empty(0, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV)
    h.sgemm_cube_token_logprobs(e, t0, v)
    x, t = logits_of(19, 4, 40, torch.float32), tokens_of(20, 4, 40)
    lp, st = torch.empty(4, device=DEV), torch.empty(4, 2, device=DEV)
    i64 = dict(dtype=torch.int64, device=DEV)
    bad = [lambda: h.sgemm_cube_token_logprobs(x, t, lp, scale=0.0), lambda: h.sgemm_cube_token_logprobs(x, t, lp, scale=-1.0),
           lambda: h.sgemm_cube_token_logprobs(x, t, lp, scale=math.inf), lambda: h.sgemm_cube_token_logprobs(x, t, lp, scale=math.nan),
           lambda: h.sgemm_cube_token_logprobs(x, None, lp),
           lambda: h.sgemm_cube_token_logprobs(x, t, lp, top_logp=torch.empty(4, 33, device=DEV), top_index=torch.empty(4, 33, **i64)),
           lambda: h.sgemm_cube_token_logprobs(x[:, :3], t, lp, top_logp=torch.empty(4, 4, device=DEV), top_index=torch.empty(4, 4, **i64)),
           lambda: h.sgemm_cube_token_logprobs(torch.empty(4, 0, device=DEV), t, lp),
           lambda: h.sgemm_cube_token_logprobs_backward(x, t, st, torch.empty_like(x)),
           lambda: h.sgemm_cube_token_logprobs_backward(x, None, st, torch.empty_like(x), dlogp=lp),
           lambda: h.sgemm_cube_token_logprobs_backward(x, t, st, torch.empty_like(x), dentropy=lp),
           lambda: h.sgemm_cube_token_logprobs_backward(x, t, None, torch.empty_like(x), dlogp=lp)]
    for call in bad:
        with pytest.raises(binding.SgemmCubeError) as err:
            call()
        assert err.value.status == binding.INVALID_ARG
    with pytest.raises(AssertionError):
        h.sgemm_cube_token_logprobs(x, t.int(), lp)
    with pytest.raises(AssertionError):
        h.sgemm_cube_token_logprobs(x.t(), t, lp)
    with pytest.raises(KeyError):
        h.sgemm_cube_token_logprobs(x.double(), t, lp)
    lib, p = binding.load(), x.data_ptr()
    assert lib.sgemm_cube_token_logprobs(h._h, 4, 40, 0, p, 39, t.data_ptr(), 1.0, lp.data_ptr(), None, None, 0, None, None, None) == binding.INVALID_ARG
    assert lib.sgemm_cube_token_logprobs(h._h, 4, 40, 7, p, 40, t.data_ptr(), 1.0, lp.data_ptr(), None, None, 0, None, None, None) == binding.INVALID_ARG
    assert lib.sgemm_cube_token_logprobs(h._h, 4, 40, 0, p + 2, 40, t.data_ptr(), 1.0, lp.data_ptr(), None, None, 0, None, None, None) == binding.INVALID_ARG
    assert lib.sgemm_cube_token_logprobs(h._h, 4, 40, 0, p, 40, t.data_ptr(), 1.0, lp.data_ptr(), None, None, 2, None, None, None) == binding.INVALID_ARG
