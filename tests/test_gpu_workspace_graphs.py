"""Captured calls go on working after larger calls on the same handle have outgrown its workspaces."""
import pytest
import torch

from paper_2507_23387_b200 import binding
from paper_2507_23387_b200.binding import ACT_GELU, WEIGHT_NK

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(seed, *shape, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV) * scale


class Step:
    """A layer with its gradients, a norm's gradients and the plain product, at one size."""

    def __init__(self, m, n, k, seed):
        self.x, self.w, self.b, self.dy = rand(seed, m, k), rand(seed + 1, n, k), rand(seed + 2, n), rand(seed + 3, m, n)
        self.mean, self.rstd, self.wt = torch.zeros(m, device=DEV), torch.ones(m, device=DEV), rand(seed + 4, k, n)
        self.y, self.z, self.c = [torch.empty(m, n, device=DEV) for _ in range(3)]
        self.dx, self.dw, self.db, self.dn = [torch.empty_like(t) for t in (self.x, self.w, self.b, self.dy)]
        self.gw, self.gb = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        self.out = [self.y, self.z, self.c, self.dx, self.dw, self.db, self.dn, self.gw, self.gb]

    def run(self, h):
        h.sgemm_cube_linear(self.x, self.w, self.y, bias=self.b, activation=ACT_GELU, preact=self.z, weight_layout=WEIGHT_NK)
        h.sgemm_cube_linear_backward(self.dy, self.x, self.w, dX=self.dx, dW=self.dw, dbias=self.db, preact=self.z,
                                     activation=ACT_GELU, weight_layout=WEIGHT_NK)
        h.sgemm_cube_layer_norm_backward(self.dy, self.y, self.mean, self.rstd, self.dn, dweight=self.gw, dbias=self.gb)
        h.sgemm_cube(self.x, self.wt, self.c)

    def results(self, run):
        for t in self.out:
            t.zero_()
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        return [t.clone() for t in self.out]


# split-K tiles and packing in one launch; several tiles with the store warps' scratch; a long contraction
SIZES = [(150, 200, 1100), (700, 520, 260), (96, 512, 4096)]


@pytest.mark.parametrize("m,n,k", SIZES)
def test_replay_after_larger_calls(m, n, k):
    h = binding.Handle(0)
    try:
        h.sgemm_cube_set_option(binding.OPT_STRATEGY, binding.STRATEGY_TWO_PHASE)
        step = Step(m, n, k, 1)
        want = step.results(lambda: step.run(h))
        assert all(torch.isfinite(t).all() and t.any() for t in want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step.run(h)
        for i, larger in enumerate(((1000, 900, 3000), (300, 4000, 5000), (2048, 4096, 4096))):
            Step(*larger, 10 * i).run(h)                      # every workspace grows, some more than once
            torch.cuda.synchronize()
            taken = [torch.full((1 << 24,), float("nan"), device=DEV) for _ in range(4)]    # whatever was given back
            got = step.results(graph.replay)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            del taken
        assert all(torch.equal(a, b) for a, b in zip(step.results(lambda: step.run(h)), want))
        assert h.sgemm_cube_check()[0] == 0
        del graph
    finally:
        h.destroy()


def test_two_graphs_of_one_handle():
    """A graph captured before and one after the growth, replayed in turn."""
    h = binding.Handle(0)
    try:
        small, large = Step(150, 200, 1100, 5), Step(900, 1000, 3000, 6)
        graphs, wants = [], []
        for s in (small, large):
            wants.append(s.results(lambda: s.run(h)))
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                s.run(h)
            graphs.append(g)
        for _ in range(2):
            for s, g, want in zip((small, large), graphs, wants):
                assert all(torch.equal(a, b) for a, b in zip(s.results(g.replay), want))
        del graphs, g
    finally:
        h.destroy()


def test_destroy_returns_outgrown_workspaces():
    def once():
        h = binding.Handle(0)
        step = Step(150, 200, 1100, 7)
        step.run(h)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step.run(h)
        Step(4096, 4096, 4096, 8).run(h)
        torch.cuda.synchronize()
        del graph
        h.destroy()
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        return torch.cuda.mem_get_info()[0]

    once()
    free = [once() for _ in range(3)]
    assert free[2] >= free[0] - (1 << 20)
