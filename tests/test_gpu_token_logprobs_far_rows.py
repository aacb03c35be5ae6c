"""Rows whose scaled logits lie on both sides of 2^25 in base 2, where the running sums change their form, against FP64.

(x - m) scale is one difference, exact for neighbouring logits, and one product; base 2 and the exponential add 2^-21 of a
term that counts, the sums of `vocab` positive terms at most (8 + vocab / 4096) u over any thread's path."""
import pytest
import torch

from paper_2507_23387_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EDGE = 2.0 ** 25 / 1.4426950408889634


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    torch.cuda.synchronize()
    handle.destroy()


def steps(x, n):
    """n representable numbers up (towards zero where x < 0) from the FP32 number nearest to x."""
    t = torch.tensor(x, dtype=torch.float32)
    for _ in range(abs(n)):
        t = torch.nextafter(t, torch.tensor(0.0 if n > 0 else -float("inf")))
    return t.item()


@pytest.mark.parametrize("scale", [1.0, 0.125, 2.0 ** 20, 3.0e7])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("vocab", [9001, 50000, 300])
@pytest.mark.parametrize("order", ["up", "down", "mixed"])
def test_both_sides_of_the_edge(h, scale, sign, vocab, order):
    levels = torch.tensor([sign * abs(steps(-EDGE / scale, n)) for n in (-3, -2, -1, 0, 1, 2)], device=DEV)
    g = torch.Generator(device=DEV).manual_seed(vocab)
    pick = torch.randint(0, 6, (6, vocab), generator=g, device=DEV)
    pick[0] = torch.arange(vocab, device=DEV) * 6 // vocab       # one level after the other
    pick[1] = (torch.arange(vocab, device=DEV) * 40 // vocab).clamp(max=5)
    if order != "mixed":
        pick[2:] = pick[2:].sort(dim=1).values
    if order == "down":
        pick = 5 - pick
    x = levels[pick]
    x[3, ::3] = -float("inf")
    x[4, ::2] = torch.finfo(torch.float32).min
    rows = x.shape[0]
    t = torch.randint(0, vocab, (rows,), generator=g, device=DEV) // 6 * 6 + 1
    t.clamp_(max=vocab - 1)
    lp, en, st = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV)
    top, index = torch.empty(rows, 5, device=DEV), torch.empty(rows, 5, dtype=torch.int64, device=DEV)
    h.sgemm_cube_token_logprobs(x, t, lp, entropy=en, stats=st, top_logp=top, top_index=index, scale=scale)
    s = torch.tensor(scale, dtype=torch.float32).double().item()
    want = torch.log_softmax(x.double() * s, 1)
    p = want.exp()
    ent = -torch.where(p > 0, p * want, torch.zeros_like(p)).sum(1)
    at = want.gather(1, t[:, None])[:, 0]
    noise = 2.0 ** -21 + (8 + vocab / 4096) * 2.0 ** -24
    ok = torch.where(at == -float("inf"), lp == at, (lp.double() - at).abs() <= noise * (1 + at.abs()))
    assert bool(ok.all()), (lp, at)
    assert bool(((en.double() - ent).abs() <= 4 * noise * (1 + ent)).all()), (en, ent)
    assert bool((st[:, 0] == x.max(1).values).all())
    first = x.double().topk(1, dim=1).values[:, 0]
    assert bool((x.gather(1, index[:, :1])[:, 0].double() == first).all())
    assert bool(((top[:, 0].double() - want.max(1).values).abs() <= noise * (1 + want.max(1).values.abs())).all())
