"""Embedding rows of more than one piece on odd addresses, and tables whose rows lie far apart."""
import pytest
import torch

from test_gpu_embedding import DEV, TYPES, gen, h, rand, want_gradient, wide  # noqa: F401  (h: the handle's fixture)

pytestmark = pytest.mark.gpu


# a piece is 128 threads x 4 vectors: 2048 FP32 or 4096 16-bit columns
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols,ld,ldy,off,offy", [(2049, 2049, 2049, 0, 0), (4097, 4099, 4101, 1, 2), (5001, 5001, 5003, 3, 0), (12295, 12295, 12295, 0, 5),
                                                  (8192, 8200, 8193, 0, 0)])
def test_lookup_and_gradient_of_wide_odd_rows(h, dtype, cols, ld, ldy, off, offy):  # noqa: F811
    rows, vocab = 37, 11
    tokens = torch.randint(0, vocab, (rows,), generator=gen(1), device=DEV)
    tokens[3], tokens[9] = -1, vocab
    table, _ = wide(vocab, cols, ld, dtype, off)
    table.copy_(rand(2, vocab, cols, dtype=dtype))
    y, buf = wide(rows, cols, ldy, dtype, offy)
    h.sgemm_cube_embedding(tokens, table, y)
    keep = (tokens >= 0) & (tokens < vocab)
    assert torch.equal(y[keep], table[tokens[keep]]) and not y[3].any() and bool(y[9].isnan().all())
    inside = torch.zeros_like(buf, dtype=torch.bool)
    torch.as_strided(inside, (rows, cols), (ldy, 1), offy).fill_(True)
    assert bool(buf[~inside].isnan().all())
    dy, _ = wide(rows, cols, ldy, dtype, offy)
    dy.copy_(rand(3, rows, cols, dtype=dtype))
    want, bound = want_gradient(tokens, dy, vocab, 1.0)
    got, buf = wide(vocab, cols, ld, torch.float32, off)
    for accumulate in (False, True):
        h.sgemm_cube_embedding_backward(tokens, dy, got, accumulate=accumulate)
        # the second call adds what is there: one more rounding of the doubled sums
        total = want * (2 if accumulate else 1)
        assert bool(((got.double() - total).abs() <= bound * (2 if accumulate else 1) + 2.0 ** -24 * total.abs() * accumulate).all())
    inside = torch.zeros_like(buf, dtype=torch.bool)
    torch.as_strided(inside, (vocab, cols), (ld, 1), off).fill_(True)
    assert bool(buf[~inside].isnan().all())


def test_no_rows_and_a_table_whose_rows_lie_gigabytes_apart(h):  # noqa: F811
    vocab, cols, ld = 3, 8, (1 << 29) + 1
    d = torch.as_strided(torch.empty((vocab - 1) * ld + cols, device=DEV), (vocab, cols), (ld, 1))
    d.fill_(3.0)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    h.sgemm_cube_embedding_backward(none, torch.empty(0, cols, device=DEV), d)
    assert not d.any()
    d.fill_(3.0)
    h.sgemm_cube_cross_entropy_backward(torch.empty(0, vocab, device=DEV), torch.ones(vocab, cols, device=DEV), none,
                                        torch.empty(0, device=DEV), dW=d)
    assert not d.any()
