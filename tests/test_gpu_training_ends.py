"""Embedding, cross entropy and orthogonalised updates together: as the example model trains with them, captured into graphs
that outlive larger calls, on other streams and on two handles at once.

Tolerance of the gradients: as in the tests of the example model, 1e-4 of a gradient's norm (one operator's result is within
2^-19 in the Frobenius norm, at most 12 operators, each enlarging what reaches it by 4 at most)."""
import subprocess
import sys

import pytest
import torch

from paper_2507_23387_b200 import binding, lm_step
from paper_2507_23387_b200.binding import WEIGHT_KN, WEIGHT_NK
from test_gpu_lm_step import loss64
from test_gpu_orthogonalize import bound, steps_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    torch.cuda.synchronize()
    handle.destroy()


def rand(seed, *shape, scale=1.0):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV) * scale


def batch(seed, tokens, vocab):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = torch.randint(0, vocab, (tokens,), generator=g, device=DEV)
    target = torch.randint(0, vocab, (tokens,), generator=g, device=DEV)
    target[1::7] = -1
    return t, target


# one row, one tile with every size odd, several tiles
@pytest.mark.parametrize("tokens,width,hidden,vocab", [(1, 64, 96, 128), (75, 97, 203, 501), (300, 256, 640, 1000)])
def test_gradients_without_logits(h, tokens, width, hidden, vocab):
    m = lm_step.Model(h, tokens + 3, width, hidden, vocab, seed=tokens, keep_logits=False)
    for i, k in enumerate(("b1", "b2", "c1", "c2", "g1", "g2")):
        m.weights[k].add_(rand(i, *m.weights[k].shape, scale=0.2))
    t, target = batch(5, tokens, vocab)
    loss = m.gradients(t, target)
    w = {k: v.double().requires_grad_(True) for k, v in m.weights.items()}
    want = loss64(w, t, target, 0.0)
    grads = dict(zip(w, torch.autograd.grad(want, list(w.values()))))
    for got in (loss, m.loss(t, target)):
        assert abs(float(got) - float(want.detach())) <= 1e-5 * max(1.0, abs(float(want.detach())))
    for k, v in grads.items():
        assert float((m.grads[k].double() - v).norm()) <= 1e-4 * float(v.norm()), k
    with pytest.raises(AssertionError):
        m.gradients(t, target, entropy_weight=0.1)
    assert h.sgemm_cube_check()[0] == 0


@pytest.mark.parametrize("width,hidden", [(96, 200), (130, 72)])
def test_step_with_orthogonal_updates(h, width, hidden):
    m = lm_step.Model(h, 60, width, hidden, 300, seed=3, keep_logits=False)
    t, target = batch(6, 50, 300)
    old = {k: v.clone() for k, v in m.weights.items()}
    rate, own, decay = 0.5, 0.02, 0.1
    m.step(t, target, rate, orthogonal=own, decay=decay)
    for k, v in m.weights.items():
        g = m.grads[k]
        if k in ("W1", "W2"):
            x = steps_of(g, torch.float64, 5)
            scale = own * max(1.0, g.shape[0] / g.shape[1]) ** 0.5
            want = (1 - own * decay) * old[k].double() - scale * x
            assert float((v.double() - want).norm()) <= bound(*g.shape, 5) * scale * float(x.norm()) + 1e-6 * float(want.norm()), k
        else:
            assert torch.equal(v, old[k] - rate * g), k


def test_runs_as_a_program():
    r = subprocess.run([sys.executable, "-m", "paper_2507_23387_b200.lm_step", "--tokens", "200", "--width", "64", "--hidden", "128",
                        "--vocab", "500", "--steps", "12", "--rate", "1.0", "--no-logits", "--orthogonal", "0.02"],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "step   11" in r.stdout and "successor" in r.stdout


class Ends:
    """The three operators at one size."""

    def __init__(self, tokens, width, vocab, other, seed, dtype=torch.float32):
        self.t, self.target = batch(seed, tokens, vocab)
        self.table, self.x = rand(seed, vocab, width).to(dtype), rand(seed + 1, tokens, width)
        self.w, self.b = rand(seed + 2, width, vocab, scale=width ** -0.5), rand(seed + 3, vocab)
        self.dloss, self.g, self.r = rand(seed + 4, tokens), rand(seed + 5, width, other), rand(seed + 6, width, other)
        self.y, self.dtable = torch.empty(tokens, width, device=DEV, dtype=dtype), torch.empty(vocab, width, device=DEV)
        self.loss, self.lse, self.few = torch.empty(tokens, device=DEV), torch.empty(tokens, device=DEV), torch.empty(3, device=DEV)
        self.dx, self.dw, self.db = torch.empty_like(self.x), torch.empty_like(self.w), torch.empty_like(self.b)
        self.o, self.o16 = torch.empty_like(self.g), torch.empty_like(self.g)
        self.out = [self.y, self.dtable, self.loss, self.lse, self.few, self.dx, self.dw, self.db, self.o, self.o16]

    def run(self, h, stream=None):
        h.sgemm_cube_embedding(self.t, self.table, self.y, stream=stream)
        h.sgemm_cube_embedding_backward(self.t, self.y, self.dtable, stream=stream)
        h.sgemm_cube_cross_entropy(self.x[:3], self.w, self.target[:3], self.few, bias=self.b, stream=stream)
        h.sgemm_cube_cross_entropy_backward(self.x, self.w, self.target, self.dloss, dX=self.dx, dW=self.dw, dbias=self.db, bias=self.b,
                                            loss=self.loss, lse=self.lse, stream=stream)
        h.sgemm_cube_orthogonalize(self.g, self.o, residual=self.r, scale=-0.1, stream=stream)
        h.sgemm_cube_orthogonalize(self.g, self.o16, steps=1, stream=stream)

    def results(self, run):
        for t in self.out:
            t.zero_()
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        return [t.clone() for t in self.out]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


# one sorting block and one piece; several of both, 16-bit rows; an update that takes a launch for every product
@pytest.mark.parametrize("args", [(30, 40, 90, 70), (5000, 65, 700, 300), (300, 2300, 400, 2400)])
def test_replay_after_larger_calls(args):
    h = binding.Handle(0)
    try:
        ends = Ends(*args, seed=1)
        want = ends.results(lambda: ends.run(h))
        assert all(torch.isfinite(t).all() and t.any() for t in want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ends.run(h)
        for i, larger in enumerate(((9000, 300, 2000, 900), (20000, 128, 60000, 4100))):
            Ends(*larger, seed=10 * i).run(h)                 # every workspace grows
            torch.cuda.synchronize()
            taken = [torch.full((1 << 24,), float("nan"), device=DEV) for _ in range(4)]    # whatever was given back
            assert same(ends.results(graph.replay), want)
            del taken
        assert same(ends.results(lambda: ends.run(h)), want)
        assert h.sgemm_cube_check()[0] == 0
        del graph
    finally:
        h.destroy()


def test_another_stream_and_two_handles_at_once():
    a, b = binding.Handle(0), binding.Handle(0)
    sizes = [(3000, 72, 900, 260), (2500, 96, 1100, 500)]
    first, second = [Ends(*s, seed=20 + i, dtype=torch.bfloat16) for i, s in enumerate(sizes)]
    want = first.results(lambda: first.run(a)), second.results(lambda: second.run(b))
    streams = [torch.cuda.Stream() for _ in range(2)]
    assert same(first.results(lambda: first.run(a, stream=streams[0])), want[0])
    with torch.cuda.stream(streams[1]):
        second.run(b)                                         # the current stream is the call's
    torch.cuda.synchronize()

    def both():
        for _ in range(5):
            first.run(a, stream=streams[0])
            second.run(b, stream=streams[1])

    got = second.results(both)
    assert same(got, want[1]) and same([t.clone() for t in first.out], want[0])
    assert a.sgemm_cube_check()[0] == 0 and b.sgemm_cube_check()[0] == 0
    a.destroy()
    b.destroy()
