"""The operators together: a training step of the small next-token model and its sampler, against FP64 autograd.

Tolerance of the gradients: one operator's result differs from its formula by at most 2^-19 in the Frobenius norm
(products: (8 + depth / 128) 2^-23 + 2^-21 at these depths; norms and probabilities less), a gradient passes
at most 12 operators, and each may enlarge what reached it by the spread of its factors, taken as 4:
12 * 4 * 2^-19 < 1e-4 of the gradient's norm."""
import subprocess
import sys

import pytest
import torch

from paper_2507_23387_b200 import binding, lm_step

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    torch.cuda.synchronize()
    handle.destroy()


def logits64(w, tokens):
    def norm(x, g, c):
        return torch.nn.functional.layer_norm(x, x.shape[-1:], g, c, 1e-5)

    x = w["E"][tokens]
    y = torch.nn.functional.gelu(norm(x, w["g1"], w["c1"]) @ w["W1"].t() + w["b1"]) @ w["W2"].t() + w["b2"] + x
    return norm(y, w["g2"], w["c2"]) @ w["H"].t()


def loss64(w, tokens, targets, entropy_weight):
    lp = torch.log_softmax(logits64(w, tokens), 1)
    known = targets >= 0
    logp = lp.gather(1, targets.clamp(min=0)[:, None])[:, 0][known]
    entropy = -(lp.exp() * lp).sum(1)[known]
    return -(logp + entropy_weight * entropy).mean()


# few rows, one tile with every size odd, several tiles
@pytest.mark.parametrize("tokens,width,hidden,vocab", [(1, 64, 96, 128), (6, 40, 104, 300), (75, 97, 203, 501), (300, 256, 640, 1000)])
@pytest.mark.parametrize("entropy_weight", [0.0, 0.1])
def test_gradients_of_every_weight(h, tokens, width, hidden, vocab, entropy_weight):
    m = lm_step.Model(h, tokens + 3, width, hidden, vocab, seed=tokens)       # room for more rows than are used
    g = torch.Generator(device=DEV).manual_seed(5)
    for k in ("b1", "b2", "c1", "c2", "g1", "g2"):
        m.weights[k].add_(torch.randn(m.weights[k].shape, generator=g, device=DEV), alpha=0.2)
    t = torch.randint(0, vocab, (tokens,), generator=g, device=DEV)
    target = torch.randint(0, vocab, (tokens,), generator=g, device=DEV)
    target[1::7] = -1
    loss = m.gradients(t, target, entropy_weight)
    w = {k: v.double().requires_grad_(True) for k, v in m.weights.items()}
    want = loss64(w, t, target, entropy_weight)
    grads = dict(zip(w, torch.autograd.grad(want, list(w.values()))))
    assert abs(float(loss) - float(want)) <= 1e-5 * max(1.0, abs(float(want)))
    for k, v in grads.items():
        assert float((m.grads[k].double() - v).norm()) <= 1e-4 * float(v.norm()), k
    assert h.sgemm_cube_check()[0] == 0


def test_training_lowers_the_loss_and_the_sampler_answers_what_was_learned(h):
    tokens, vocab = 256, 512
    m = lm_step.Model(h, tokens, 128, 256, vocab, seed=1)
    g = torch.Generator(device=DEV).manual_seed(2)
    successor = torch.randperm(vocab, generator=g, device=DEV)
    t = torch.randperm(vocab, generator=g, device=DEV)[:tokens]
    losses = [float(m.step(t, successor[t], 2.0)) for _ in range(60)]
    assert losses[-1] < 0.25 * losses[0]
    s = lm_step.Sampler(m, 12, top=4)
    for n in (1, 7, 12):
        logp, top = s.next(t[:n], temperature=0.5)
        want, index = torch.log_softmax(2.0 * logits64({k: v.double() for k, v in m.weights.items()}, t[:n]), 1).topk(4)
        # logits of size 10 off by 1e-5 of that at most, twice (scale), in the value and in the sum
        assert bool(((logp.double() - want).abs() <= 4e-4).all())
        assert torch.equal(top[:, 0], index[:, 0])
        assert float((top[:, 0] == successor[t[:n]]).float().mean()) > 0.5
    allowed = torch.zeros(vocab, dtype=torch.bool, device=DEV)
    logp, _ = s.next(t[:3], allowed=allowed)
    assert bool((logp == float("-inf")).all())
    allowed[7] = True
    logp, top = s.next(t[:3], allowed=allowed)
    assert bool((logp[:, 0] == 0).all()) and bool((top[:, 0] == 7).all()) and bool((logp[:, 1:] == float("-inf")).all())


def test_runs_as_a_program():
    r = subprocess.run([sys.executable, "-m", "paper_2507_23387_b200.lm_step", "--tokens", "200", "--width", "64", "--hidden", "128",
                        "--vocab", "500", "--steps", "12", "--rate", "1.0"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "step   11" in r.stdout and "successor" in r.stdout
