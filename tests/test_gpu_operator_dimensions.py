"""Dimensions above 2^31 - 2^16 are refused on the host, before any launch: the kernels count in 32 bits and step past
the end of a row by a block's stride."""
import pytest
import torch

from paper_2507_23387_b200 import binding
from paper_2507_23387_b200.binding import INVALID_ARG

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LIMIT = 2 ** 31 - 2 ** 16


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    handle.destroy()


@pytest.mark.parametrize("d", [LIMIT + 1, 2 ** 31 - 1, -1])
def test_dimensions(h, d):
    lib, big = binding.load(), 2 ** 40
    before = h.sgemm_cube_launch_count()
    f, t = torch.zeros(64, device=DEV).data_ptr(), torch.zeros(8, device=DEV, dtype=torch.int64).data_ptr()
    o = binding._Operand(f, big, None, None, 0, None)
    for rows, cols in ((d, 1), (1, d)):
        assert lib.sgemm_cube_pack(h._h, rows, cols, f, big, f, f, big, f, None) == INVALID_ARG
        assert lib.sgemm_cube_layer_norm(h._h, rows, cols, 0, f, big, None, None, 1e-5, f, big, None, None, None) == INVALID_ARG
        assert lib.sgemm_cube_layer_norm_backward(h._h, rows, cols, 0, f, big, f, big, None, f, f, f, big, f, f, None) == INVALID_ARG
        assert lib.sgemm_cube_token_logprobs(h._h, rows, cols, 0, f, big, t, 1.0, f, None, None, 0, None, None, None) == INVALID_ARG
        assert lib.sgemm_cube_token_logprobs_backward(h._h, rows, cols, 0, f, big, t, 1.0, f, None, f, None, f, big, None) == INVALID_ARG
    for m, n, k in ((d, 1, 1), (1, d, 1), (1, 1, d)):
        for layout in (0, 1):
            assert lib.sgemm_cube_linear(h._h, m, n, k, o, o, layout, None, None, 0, 0, f, big, None, 0, None) == INVALID_ARG
            assert lib.sgemm_cube_linear_backward(h._h, m, n, k, f, big, None, 0, 0, o, o, layout, f, big, f, big, f, None) == INVALID_ARG
    assert h.sgemm_cube_launch_count() == before


def test_many_rows_of_one_column(h):
    """Hundreds of millions of rows: the gradient of one output's bias, and rows of one element.  A warp's halves add up
    exactly; some 1200 partial sums follow, one rounding each."""
    m = 300_000_001
    dy, db = torch.full((m, 1), 0.5, device=DEV), torch.empty(1, device=DEV)
    x, w = torch.empty(m, 1, device=DEV), torch.empty(1, 1, device=DEV)
    h.sgemm_cube_linear_backward(dy, x, w, dbias=db)
    assert abs(float(db) / (0.5 * m) - 1) <= 1300 * 2.0 ** -24
    y = torch.full((m, 1), 9.0, device=DEV)
    h.sgemm_cube_layer_norm(dy, y)
    assert float(y.abs().max()) == 0.0
    t, lp = torch.zeros(m, dtype=torch.int64, device=DEV), torch.full((m,), 9.0, device=DEV)
    h.sgemm_cube_token_logprobs(dy, t, lp)
    assert float(lp.abs().max()) == 0.0
