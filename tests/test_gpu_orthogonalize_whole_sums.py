"""Orthogonalised updates under the option that keeps sums whole: one launch for all products then leaves their k ranges whole, too.

Bounds: those of the polynomial in 64 bits."""
import pytest
import torch

from paper_2507_23387_b200 import binding
from test_gpu_orthogonalize import check, rand

pytestmark = pytest.mark.gpu


# few tiles under long sums, which are cut along k by default
@pytest.mark.parametrize("rows,cols", [(128, 8000), (8000, 128), (300, 5001), (7, 9001)])
def test_option_reaches_the_one_launch(rows, cols):
    h = binding.Handle(0)
    g = rand(rows, rows, cols)
    cut = check(h, g, 1)
    h.sgemm_cube_set_option(binding.OPT_SPLIT_K, 0)
    before = h.sgemm_cube_launch_count()
    whole = check(h, g, 1)
    assert h.sgemm_cube_launch_count() - before == 1
    check(h, g, 5)
    # the same sums in another order: some of the many entries are rounded otherwise
    assert not torch.equal(whole, cut)
    h.sgemm_cube_set_option(binding.OPT_SPLIT_K, 1)
    assert torch.equal(check(h, g, 1), cut)
    assert h.sgemm_cube_check()[0] == 0
    h.destroy()
