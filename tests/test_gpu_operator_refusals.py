"""What the language-model operators refuse by pointer and place, on the host and before any launch: addresses that
are not a multiple of the element's size, and results in the place of an operand that they may not take."""
import pytest
import torch

from paper_2507_23387_b200 import binding
from paper_2507_23387_b200.binding import INVALID_ARG, PackedMatrix

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    torch.cuda.synchronize()
    assert handle.sgemm_cube_check()[0] == 0
    handle.destroy()


def room(*shape, dtype=torch.float32):
    return torch.ones(shape, device=DEV, dtype=dtype)


def every_shift(call, args, size):
    """The call with each of the pointers moved by a part of its element; unmoved it is accepted."""
    assert call(**args) == 0
    for name in args:
        for by in {1, size // 2, size - 1} - {0}:
            assert call(**{**args, name: args[name] + by}) == INVALID_ARG, (name, by)


def fp32(p, ld):
    return binding._Operand(p, ld, None, None, 0, None)


def test_linear(h):
    lib, m, n, k = binding.load(), 5, 6, 8
    t = dict(x=room(m, k), w=room(k, n), bias=room(n), r=room(m, n), y=room(m, n), z=room(m, n))
    before = h.sgemm_cube_launch_count()

    def forward(x, w, bias, r, y, z, ldr=n, rows=m):
        return lib.sgemm_cube_linear(h._h, rows, n, k, fp32(x, k), fp32(w, n), 0, bias, r, ldr, 1, y, n, z, n, None)

    args = {name: v.data_ptr() for name, v in t.items()}
    every_shift(forward, args, 4)
    assert forward(**{**args, "z": args["y"]}) == INVALID_ARG and forward(**{**args, "z": args["r"]}) == INVALID_ARG
    assert forward(**{**args, "r": args["y"]}) == 0
    assert forward(**{**args, "r": args["y"]}, ldr=n + 1) == INVALID_ARG
    assert forward(**{**args, "r": args["y"]}, ldr=n + 1, rows=1) == 0         # one row has no leading dimension
    torch.cuda.synchronize()
    accepted = h.sgemm_cube_launch_count() - before
    assert accepted > 0
    t = dict(dy=room(m, n), z=room(m, n), x=room(m, k), w=room(k, n), dx=room(m, k), dw=room(k, n), db=room(n))

    def backward(dy, z, x, w, dx, dw, db):
        return lib.sgemm_cube_linear_backward(h._h, m, n, k, dy, n, z, n, 1, fp32(x, k), fp32(w, n), 0, dx, k, dw, n, db, None)

    every_shift(backward, {name: v.data_ptr() for name, v in t.items()}, 4)


def test_pack(h):
    lib, x, p = binding.load(), room(7, 9), PackedMatrix(7, 9)
    o = p.operand

    def pack(x, exp):
        return lib.sgemm_cube_pack(h._h, 7, 9, x, 9, o.hi_dev, o.lo_dev, o.ld16, exp, None)

    every_shift(pack, dict(x=x.data_ptr(), exp=o.exp_dev), 4)
    y, a = room(4, 7), room(4, 9)

    def packed(exp):
        w = binding._Operand(None, 0, o.hi_dev, o.lo_dev, o.ld16, exp)
        return lib.sgemm_cube_linear(h._h, 4, 7, 9, fp32(a.data_ptr(), 9), w, 1, None, None, 0, 0, y.data_ptr(), 7, None, 0, None)

    every_shift(packed, dict(exp=o.exp_dev), 4)


@pytest.mark.parametrize("dtype,code", [(torch.float32, 0), (torch.float16, 1), (torch.bfloat16, 2)])
def test_layer_norm(h, dtype, code):
    lib, rows, cols = binding.load(), 5, 24
    x, y, g, dx = [room(rows, cols, dtype=dtype) for _ in range(4)]
    v = dict(weight=room(cols), bias=room(cols), mean=room(rows), rstd=room(rows))

    def forward(x, y, weight=None, bias=None, mean=None, rstd=None, ldy=cols, rows=rows):
        return lib.sgemm_cube_layer_norm(h._h, rows, cols, code, x, cols, weight, bias, 1e-5, y, ldy, mean, rstd, None)

    px, py, pg, pdx = [t.data_ptr() for t in (x, y, g, dx)]
    every_shift(lambda x, y: forward(x, y), dict(x=px, y=py), x.element_size())
    every_shift(lambda **kw: forward(px, py, **kw), {n: t.data_ptr() for n, t in v.items()}, 4)
    assert forward(px, px) == 0 and forward(px, px, ldy=cols + 8) == INVALID_ARG
    assert forward(px, px, ldy=cols + 8, rows=1) == 0
    v = dict(weight=room(cols), mean=room(rows), rstd=room(rows), dweight=room(cols), dbias=room(cols))

    def backward(dy, x, dx, weight=None, mean=v["mean"].data_ptr(), rstd=v["rstd"].data_ptr(), dweight=None, dbias=None, lddx=cols):
        return lib.sgemm_cube_layer_norm_backward(h._h, rows, cols, code, dy, cols, x, cols, weight, mean, rstd, dx, lddx,
                                                  dweight, dbias, None)

    every_shift(lambda dy, x, dx: backward(dy, x, dx), dict(dy=pg, x=px, dx=pdx), x.element_size())
    every_shift(lambda **kw: backward(pg, px, pdx, **kw), {n: t.data_ptr() for n, t in v.items()}, 4)
    assert backward(pg, px, pg, lddx=cols + 8) == INVALID_ARG
    assert backward(pg, px, pg) == 0


@pytest.mark.parametrize("dtype,code", [(torch.float32, 0), (torch.float16, 1), (torch.bfloat16, 2)])
def test_token_logprobs(h, dtype, code):
    lib, rows, vocab, k = binding.load(), 4, 40, 3
    x, dx, tokens, index = room(rows, vocab, dtype=dtype), room(rows, vocab, dtype=dtype), room(rows, dtype=torch.int64), \
        room(rows, k, dtype=torch.int64)
    v = dict(logp=room(rows), entropy=room(rows), stats=room(rows, 2), top=room(rows, k))
    f = {n: t.data_ptr() for n, t in v.items()}
    px, pt, pi, pdx = [t.data_ptr() for t in (x, tokens, index, dx)]

    def forward(x=px, tokens=pt, index=pi, logp=f["logp"], entropy=f["entropy"], stats=f["stats"], top=f["top"]):
        return lib.sgemm_cube_token_logprobs(h._h, rows, vocab, code, x, vocab, tokens, 1.0, logp, entropy, stats, k, top, index, None)

    every_shift(forward, dict(x=px), x.element_size())
    every_shift(forward, dict(tokens=pt, index=pi), 8)
    every_shift(forward, f, 4)
    g = dict(stats=f["stats"], entropy=f["entropy"], dlogp=room(rows).data_ptr(), dentropy=f["logp"])

    def backward(x=px, tokens=pt, dx=pdx, stats=g["stats"], entropy=g["entropy"], dlogp=g["dlogp"], dentropy=g["dentropy"], lddl=vocab):
        return lib.sgemm_cube_token_logprobs_backward(h._h, rows, vocab, code, x, vocab, tokens, 1.0, stats, entropy, dlogp,
                                                      dentropy, dx, lddl, None)

    every_shift(backward, dict(x=px, dx=pdx), x.element_size())
    every_shift(backward, dict(tokens=pt), 8)
    every_shift(backward, g, 4)
    assert backward(dx=px, lddl=vocab + 8) == INVALID_ARG
    assert backward(dx=px) == 0
