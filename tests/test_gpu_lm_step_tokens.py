"""Tokens as the example model has always taken them: 32-bit ones and views of a larger tensor, in every call that embeds."""
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
    assert handle.sgemm_cube_check()[0] == 0
    handle.destroy()


def columns(tokens):
    """The same tokens, every second of another tensor's."""
    return torch.stack((tokens, torch.zeros_like(tokens)), 1)[:, 0]


@pytest.mark.parametrize("form", [lambda t: t.int(), columns, lambda t: columns(t.int())])
@pytest.mark.parametrize("keep_logits", [True, False])
def test_training_takes_tokens_of_either_width_and_stride(h, form, keep_logits):
    g = torch.Generator(device=DEV).manual_seed(1)
    tokens = torch.randint(0, 300, (40,), generator=g, device=DEV)
    targets = torch.randint(0, 300, (40,), generator=g, device=DEV)
    a, b = [lm_step.Model(h, 40, 64, 96, 300, seed=2, keep_logits=keep_logits) for _ in range(2)]
    assert torch.equal(a.loss(tokens, targets), b.loss(form(tokens), targets))
    if keep_logits:
        assert torch.equal(a.forward(tokens, targets)["logp"], b.forward(form(tokens), targets)["logp"])
    assert torch.equal(a.step(tokens, targets, 0.5), b.step(form(tokens), targets, 0.5))
    for k in a.weights:
        assert torch.equal(a.grads[k], b.grads[k]) and torch.equal(a.weights[k], b.weights[k]), k


@pytest.mark.parametrize("form", [lambda t: t.int(), columns])
def test_sampling_takes_tokens_of_either_width_and_stride(h, form):
    s = lm_step.Sampler(lm_step.Model(h, 8, 64, 96, 300, seed=3), 8)
    tokens = torch.tensor([5, 0, 299, 5, 77], device=DEV)
    want = [t.clone() for t in s.next(tokens)]
    for got, w in zip(s.next(form(tokens)), want):
        assert torch.equal(got, w)
