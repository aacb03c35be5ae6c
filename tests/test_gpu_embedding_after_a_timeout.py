"""The table's gradient behind a sort whose blocks did not meet (a count left on the handle lets them all pass): whatever the
workspace holds, nothing outside the operands is touched, the status is reported, and the next gradient is right."""
import pytest
import torch

from paper_2507_23387_b200 import binding
from test_gpu_embedding import DEV, TYPES, rand, tokens_like_text, want_gradient, wide

pytestmark = pytest.mark.gpu
SORT_CODE = 0x10C


# more rows than are ranked without meetings; one, two and three passes over the digits
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,cols", [(20000, 100, 40), (9001, 3000, 17), (40000, 300000, 12)])
def test_stays_within_its_operands_and_recovers(dtype, rows, vocab, cols):
    h = binding.Handle(0)
    # a larger call's tokens and rows, none of them this call's, are what the workspace holds
    big = torch.arange(400000, device=DEV) % 390000
    h.sgemm_cube_embedding_backward(big, rand(1, 400000, 4, dtype=dtype), torch.empty(390000, 4, device=DEV))
    assert h.sgemm_cube_check() == (0, 0)
    tokens, dy = tokens_like_text(2, rows, vocab), rand(3, rows, cols, dtype=dtype)
    got, buf = wide(vocab, cols, cols + 4, offset=1024)
    outside = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(outside, (vocab, cols), (cols + 4, 1), 1024).fill_(False)
    kept = tokens.clone(), dy.clone()
    for accumulate in (False, True):
        h.sgemm_cube_debug_inject_error(SORT_CODE)
        h.sgemm_cube_embedding_backward(tokens, dy, got, accumulate=accumulate)
        assert h.sgemm_cube_check() == (binding.DEVICE_TIMEOUT, SORT_CODE)
        assert bool(buf[outside].isnan().all()) and torch.equal(tokens, kept[0]) and torch.equal(dy, kept[1])
    want, bound = want_gradient(tokens, dy, vocab, 1.0)
    h.sgemm_cube_embedding_backward(tokens, dy, got)
    assert bool(((got.double() - want).abs() <= bound).all())
    assert h.sgemm_cube_check() == (0, 0)
    h.destroy()
