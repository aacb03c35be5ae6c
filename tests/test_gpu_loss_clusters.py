"""A row's loss from logits that a cluster of blocks shares: the same to the bit however the blocks of the cluster come to run,
one call alone, many calls behind one another, and calls beside others that keep most of the SMs busy."""
import pytest
import torch

from paper_2507_23387_b200 import binding
from test_gpu_cross_entropy import DEV, Case

pytestmark = pytest.mark.gpu


# two, four and eight blocks a row, the least work of each; one row of eight and as many as share the SMs
@pytest.mark.parametrize("m,n", [(1, 8192), (3, 16384), (1, 32768), (4, 40001), (40, 65536)])
def test_rows_of_a_cluster_beside_other_work(m, n):
    h = binding.Handle(0)
    c = Case(m, n, 16, binding.WEIGHT_NK, seed=m)
    want = [t.clone() for t in c.check_forward(h)]
    side = torch.cuda.Stream()
    busy = [torch.randn(2048, 2048, device=DEV) for _ in range(3)]
    runs = 60
    loss, lse = torch.full((runs, m), float("nan"), device=DEV), torch.full((runs, m), float("nan"), device=DEV)
    torch.cuda.synchronize()
    for beside in (False, True):
        loss.fill_(float("nan"))
        lse.fill_(float("nan"))
        torch.cuda.synchronize()
        for i in range(runs):
            if beside and i % 6 == 0:
                with torch.cuda.stream(side):
                    torch.matmul(busy[0], busy[1], out=busy[2])
            h.sgemm_cube_cross_entropy(c.x, c.w, c.targets, loss[i], bias=c.bias, lse=lse[i], weight_layout=c.layout)
        torch.cuda.synchronize()
        assert bool((loss == want[0]).all()) and bool((lse == want[1]).all())
    assert h.sgemm_cube_check()[0] == 0
    h.destroy()
