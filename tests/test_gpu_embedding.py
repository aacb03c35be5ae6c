"""Embedding lookup and the table's gradient against 64-bit sums, over element types, strides, odd widths and token counts on
both sides of what one sorting block, one piece of the sorted rows and one pass over the digits hold."""
import pytest
import torch

from paper_2507_23387_b200 import binding
from paper_2507_23387_b200.binding import INVALID_ARG

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    torch.cuda.synchronize()
    assert handle.sgemm_cube_check()[0] == 0
    handle.destroy()


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rand(seed, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen(seed), device=DEV).to(dtype)


def fp32(x):
    """The scale as the call takes it: FP32, up to 2^-24 of itself from the number written here."""
    return torch.tensor(x, dtype=torch.float32).item()


def wide(rows, cols, ld, dtype=torch.float32, offset=0):
    """A rows x cols view with a leading dimension of ld, `offset` elements behind an aligned address; NaN around it."""
    buf = torch.full((rows * ld + offset,), float("nan"), device=DEV, dtype=dtype)
    return torch.as_strided(buf, (rows, cols), (ld, 1), offset), buf


def want_gradient(tokens, dy, vocab, scale):
    """FP64 sums, and the bound of FP32 ones: every addition and the scaling off by 2^-24 of what has been added."""
    keep = (tokens >= 0) & (tokens < vocab)
    t, d = tokens[keep], dy[keep].double()
    zero = torch.zeros(vocab, dy.shape[1], dtype=torch.float64, device=DEV)
    sums, mags = zero.clone().index_add_(0, t, d) * fp32(scale), zero.index_add_(0, t, d.abs()) * abs(fp32(scale))
    count = torch.bincount(t, minlength=vocab)[:, None].double()
    return sums, (count + 2) * U * mags


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,cols,scale", [(1, 1, 1, 1.0), (5, 3, 8, -2.5), (17, 300, 129, 1.0), (3, 1000, 4096, 64.0),
                                                   (700, 65, 2056, 0.3), (260, 7, 515, 1.0)])
def test_lookup(h, dtype, rows, vocab, cols, scale):
    table, tokens = rand(1, vocab, cols, dtype=dtype), torch.randint(0, vocab, (rows,), generator=gen(2), device=DEV)
    y = torch.full((rows, cols), float("nan"), device=DEV, dtype=dtype)
    h.sgemm_cube_embedding(tokens, table, y, scale=scale)
    want = table[tokens].double() * fp32(scale)
    # one FP32 product, one rounding to the type (half a step; FP16 subnormals 2^-25)
    half = 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2
    assert bool(((y.double() - want).abs() <= (half + U) * 1.01 * want.abs() + 2.0 ** -25 * (dtype == torch.float16)).all())
    if scale == 1.0:
        assert torch.equal(y, table[tokens])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols,ld,ldy,off", [(24, 24, 32, 0), (24, 25, 24, 1), (17, 40, 19, 3), (640, 648, 648, 8)])
def test_lookup_strides_padding_and_unknown_tokens(h, dtype, cols, ld, ldy, off):
    vocab, tokens = 50, torch.tensor([3, -1, 49, 50, 0, 2 ** 40, -2 ** 60, 3], device=DEV)
    table, _ = wide(vocab, cols, ld, dtype, off)
    table.copy_(rand(3, vocab, cols, dtype=dtype))
    y, buf = wide(8, cols, ldy, dtype, off)
    before = buf.clone()
    h.sgemm_cube_embedding(tokens, table, y)
    for i, t in enumerate(tokens.tolist()):
        if t < 0:
            assert bool((y[i] == 0).all())
        elif t >= vocab:
            assert bool(torch.isnan(y[i]).all())
        else:
            assert torch.equal(y[i], table[t])
    inside = torch.zeros_like(buf, dtype=torch.bool)
    torch.as_strided(inside, (8, cols), (ldy, 1), off).fill_(True)
    assert bool(torch.isnan(buf[~inside]).all()) and bool(torch.isnan(before).all())


def tokens_like_text(seed, rows, vocab):
    return (torch.rand(rows, generator=gen(seed), device=DEV, dtype=torch.float64) ** 4 * vocab).long().clamp_(max=vocab - 1)


# one row; a piece; several pieces; more than a sorting block; two and three passes over the digits; several columns tiles
SIZES = [(1, 1, 1), (2, 300, 40), (31, 10, 7), (33, 5, 129), (700, 255, 520), (2049, 256, 36), (5000, 70000, 24), (9001, 40, 1030),
         (40000, 1001, 17), (300000, 200000, 4)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,cols", SIZES)
def test_gradient(h, dtype, rows, vocab, cols):
    tokens, dy, scale = tokens_like_text(4, rows, vocab), rand(5, rows, cols, dtype=dtype), 0.7
    if rows > 8:
        tokens[3::11] = -1
        tokens[5::17] = vocab + 3
    want, bound = want_gradient(tokens, dy, vocab, scale)
    got = torch.full((vocab, cols), float("nan"), device=DEV)
    h.sgemm_cube_embedding_backward(tokens, dy, got, scale=scale)
    assert bool(((got.double() - want).abs() <= bound).all())
    again = torch.empty_like(got)
    h.sgemm_cube_embedding_backward(tokens, dy, again, scale=scale)
    assert torch.equal(got, again)
    base = rand(6, vocab, cols)
    held = base.clone()
    h.sgemm_cube_embedding_backward(tokens, dy, held, scale=scale, accumulate=True)
    assert bool(((held.double() - base.double() - want).abs() <= bound + U * (base.double().abs() + want.abs() + bound)).all())
    unmet = torch.ones(vocab, dtype=torch.bool, device=DEV)
    unmet[tokens[(tokens >= 0) & (tokens < vocab)]] = False
    assert torch.equal(held[unmet], base[unmet]) and bool((got[unmet] == 0).all())


@pytest.mark.parametrize("rows", [1, 31, 32, 33, 64, 1000, 5000])
def test_gradient_of_one_token_alone_and_among_padding(h, rows):
    """A run that fills every piece, with nothing around it and behind unknown tokens."""
    dy = rand(7, rows, 12)
    for tokens in (torch.full((rows,), 2, device=DEV), torch.full((rows,), -1, device=DEV)):
        tokens = tokens.clone()
        tokens[::5] = 2
        want, bound = want_gradient(tokens, dy, 4, 1.0)
        got = torch.empty(4, 12, device=DEV)
        h.sgemm_cube_embedding_backward(tokens, dy, got)
        assert bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols,ldy,ldd,off", [(24, 24, 40, 0), (24, 25, 27, 1), (17, 18, 33, 3), (520, 528, 524, 4)])
def test_gradient_strides(h, dtype, cols, ldy, ldd, off):
    rows, vocab = 100, 30
    tokens = tokens_like_text(8, rows, vocab)
    dy, _ = wide(rows, cols, ldy, dtype, off)
    dy.copy_(rand(9, rows, cols, dtype=dtype))
    got, buf = wide(vocab, cols, ldd, torch.float32, off)
    h.sgemm_cube_embedding_backward(tokens, dy, got)
    want, bound = want_gradient(tokens, dy, vocab, 1.0)
    assert bool(((got.double() - want).abs() <= bound).all())
    inside = torch.zeros_like(buf, dtype=torch.bool)
    torch.as_strided(inside, (vocab, cols), (ldd, 1), off).fill_(True)
    assert bool(torch.isnan(buf[~inside]).all())


@pytest.mark.parametrize("vocab,cols,ldd,off", [(41, 4096, 4096, 0), (41, 4096, 4096, 1), (3, 20000, 20000, 31), (3, 20000, 20003, 17),
                                                (4096, 12, 12, 32), (9001, 5, 5, 7), (1000, 33, 40, 3), (1, 1, 1, 5), (130, 127, 127, 30)])
@pytest.mark.parametrize("met", ["none", "few", "ends", "every other"])
def test_rows_without_tokens_are_zeros_and_nothing_else_is_written(h, vocab, cols, ldd, off, met):
    """Zeros go out in pieces that begin at their own addresses, inside rows and across them."""
    tokens = {"none": torch.tensor([-1, vocab]), "few": torch.tensor([vocab // 2, vocab // 3, vocab // 2]),
              "ends": torch.tensor([0, vocab - 1]), "every other": torch.arange(0, vocab, 2)}[met].to(DEV)
    dy = torch.ones(len(tokens), cols, device=DEV)
    grad, buf = wide(vocab, cols, ldd, offset=off)
    h.sgemm_cube_embedding_backward(tokens, dy, grad)
    keep = tokens[(tokens >= 0) & (tokens < vocab)]
    assert torch.equal(grad, torch.bincount(keep, minlength=vocab).float()[:, None].expand(vocab, cols))
    inside = torch.zeros(len(buf), dtype=torch.bool, device=DEV)
    torch.as_strided(inside, (vocab, cols), (ldd, 1), off).fill_(True)
    assert bool(buf[~inside].isnan().all())


@pytest.mark.parametrize("rows", [255, 256, 257, 383, 385, 1023, 1025, 2047, 4099, 8191, 8192, 8193])
@pytest.mark.parametrize("vocab", [1, 3, 700, 300000])
def test_gradient_on_both_sides_of_what_is_ranked_and_sorted(h, rows, vocab):
    tokens, dy = tokens_like_text(31, rows, vocab), rand(32, rows, 12)
    tokens[::7] = vocab
    tokens[rows // 2:rows // 2 + 40] = -1
    tokens[-1] = vocab - 1
    want, bound = want_gradient(tokens, dy, vocab, 1.0)
    got = torch.full((vocab, 12), float("nan"), device=DEV)
    for accumulate in (False, True):
        h.sgemm_cube_embedding_backward(tokens, dy, got, accumulate=accumulate)
        # the second call adds what is there: one more rounding of the doubled sums
        total = want * (2 if accumulate else 1)
        assert bool(((got.double() - total).abs() <= bound * (2 if accumulate else 1) + U * total.abs() * accumulate).all())


def test_gradient_of_infinite_rows_stays_in_their_tokens(h):
    rows, cols = 200, 9
    tokens, dy = torch.arange(rows, device=DEV) % 20, rand(10, rows, cols)
    dy[7, 3], dy[40, 1] = float("inf"), float("nan")
    got = torch.empty(20, cols, device=DEV)
    h.sgemm_cube_embedding_backward(tokens, dy, got)
    bad = ~torch.isfinite(got)
    assert bad.sum() == 2 and bool(bad[7, 3]) and bool(bad[0, 1])


def test_no_rows(h):
    none, d = torch.empty(0, dtype=torch.int64, device=DEV), torch.full((5, 6), 3.0, device=DEV)
    h.sgemm_cube_embedding(none, d, torch.empty(0, 6, device=DEV))
    h.sgemm_cube_embedding_backward(none, torch.empty(0, 6, device=DEV), d, accumulate=True)
    assert bool((d == 3.0).all())
    h.sgemm_cube_embedding_backward(none, torch.empty(0, 6, device=DEV), d)
    assert bool((d == 0.0).all())


def test_offsets_past_32_bits(h):
    vocab, cols, ld = 5, 1000, 540_000_000
    table, _ = torch.as_strided(torch.empty((vocab - 1) * ld + cols, device=DEV), (vocab, cols), (ld, 1)), None
    table.copy_(rand(11, vocab, cols))
    tokens, y = torch.tensor([4, 0, 3, 4], device=DEV), torch.empty(4, cols, device=DEV)
    h.sgemm_cube_embedding(tokens, table, y)
    assert torch.equal(y, table[tokens])
    want, bound = want_gradient(tokens, y, vocab, 1.0)
    h.sgemm_cube_embedding_backward(tokens, y, table)
    assert bool(((table.double() - want).abs() <= bound).all())


def test_refusals(h):
    lib, rows, vocab, cols = binding.load(), 4, 6, 8
    tokens, table, y = torch.zeros(rows, dtype=torch.int64, device=DEV), torch.ones(vocab, cols, device=DEV), torch.ones(rows, cols, device=DEV)
    pt, pe, py = tokens.data_ptr(), table.data_ptr(), y.data_ptr()

    def look(rows=rows, vocab=vocab, cols=cols, dtype=0, t=pt, e=pe, ld=cols, s=1.0, y=py, ldy=cols):
        return lib.sgemm_cube_embedding(h._h, rows, vocab, cols, dtype, t, e, ld, s, y, ldy, None)

    def back(rows=rows, vocab=vocab, cols=cols, dtype=0, t=pt, g=py, ldg=cols, s=1.0, acc=0, d=pe, ldd=cols):
        return lib.sgemm_cube_embedding_backward(h._h, rows, vocab, cols, dtype, t, g, ldg, s, acc, d, ldd, None)

    assert look() == 0 and back() == 0
    before = h.sgemm_cube_launch_count()
    for bad in (dict(rows=-1), dict(rows=2 ** 31 - 1), dict(vocab=0), dict(vocab=2 ** 31 - 1), dict(cols=0), dict(dtype=3), dict(dtype=-1),
                dict(t=None), dict(t=pt + 4), dict(s=float("nan")), dict(s=float("inf"))):
        assert look(**bad) == INVALID_ARG, bad
        assert back(**bad) == INVALID_ARG, bad
    for bad in (dict(e=None), dict(y=None), dict(e=pe + 1), dict(y=py + 2), dict(ld=cols - 1), dict(ldy=cols - 1), dict(y=pe)):
        assert look(**bad) == INVALID_ARG, bad
    for bad in (dict(g=None), dict(d=None), dict(g=py + 2), dict(d=pe + 2), dict(ldg=cols - 1), dict(ldd=cols - 1), dict(acc=2)):
        assert back(**bad) == INVALID_ARG, bad
    assert h.sgemm_cube_launch_count() == before
