"""Cross entropy without the logits, and its gradients, against the definition in 64 bits.

Bounds.  u = 2^-24.  A logit is off by E = 1.2 max(2 K, K + 14) u (|x| |w|) + u |z| (the product's bound, and the bias).  In a
row the largest of these moves lse by no more than itself and the loss by no more than twice that.  The sum of exponentials
adds at most 200 u: exponents are off by 3 u |z - m|, 72 u where that averages 24 (a vocabulary of 10^5), the exponential 4 u,
additions and the joining of 64 columns' pairs 40 and 64 u.  The loss' own operations: 4 u of its terms.
dz is off by that share of |dloss| (p + 1[t]), its words by 2^-21; the gradients' products by the product's bound."""
import pytest
import torch

from paper_2507_23387_b200 import binding
from paper_2507_23387_b200.binding import INVALID_ARG, MISALIGNED, WEIGHT_KN, WEIGHT_NK, PackedMatrix

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(0)
    yield handle
    torch.cuda.synchronize()
    assert handle.sgemm_cube_check()[0] == 0
    handle.destroy()


def rand(seed, *shape, scale=1.0):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV) * scale


def product_bound(k):
    return 1.2 * max(2 * k, k + 14) * U


class Case:
    """Inputs, the 64-bit results and their bounds."""

    def __init__(self, m, n, k, layout, bias=True, seed=0, scale=2.0):
        self.m, self.n, self.k, self.layout = m, n, k, layout
        self.w = rand(seed, *((n, k) if layout == WEIGHT_NK else (k, n)), scale=scale * k ** -0.5)
        self.x = rand(seed + 1, m, k)
        self.bias = rand(seed + 2, n) if bias else None
        g = torch.Generator(device=DEV).manual_seed(seed + 3)
        self.targets = torch.randint(0, n, (m,), generator=g, device=DEV)
        if m > 3:
            self.targets[1::5] = -1
        self.dloss = rand(seed + 4, m, scale=1.0 / m)
        self.targets64()

    def targets64(self):
        w = (self.w.t() if self.layout == WEIGHT_NK else self.w).double()
        x = self.x.double()
        z = x @ w + (0 if self.bias is None else self.bias.double())
        row = product_bound(self.k) * (x.abs() @ w.abs()) + U * z.abs()
        self.off = torch.where(torch.isfinite(z), row, 0.0).amax(1) + 200 * U       # of a row's logits
        self.lse = torch.logsumexp(z, 1)
        known = self.targets >= 0
        at = self.targets.clamp(min=0)[:, None]
        zt, top = z.gather(1, at)[:, 0], z.amax(1)
        self.loss = torch.where(known, self.lse - zt, 0.0)
        self.lse_bound = self.off + 4 * U * (self.lse.abs() + top.abs())
        self.loss_bound = 2 * self.off + 4 * U * (self.loss.abs() + (top - zt).abs())
        p = torch.exp(z - self.lse[:, None])
        hot = torch.zeros_like(p).scatter_(1, at, 1.0)
        d = torch.where(known, self.dloss.double(), 0.0)[:, None]
        self.dz, mag = d * (p - hot), d.abs() * (p + hot)
        rel = 2 * self.off.max() + 2.0 ** -21
        self.dx, self.dw, self.db = self.dz @ w.t(), x.t() @ self.dz, self.dz.sum(0)
        # (a column's sum: m additions, in FP32)
        self.dx_bound = (rel + product_bound(self.n)) * (mag @ w.abs().t())
        self.dw_bound = (rel + product_bound(self.m)) * (x.abs().t() @ mag)
        self.db_bound = (rel + (self.m + 8) * U) * mag.sum(0)
        if self.layout == WEIGHT_NK:
            self.dw, self.dw_bound = self.dw.t(), self.dw_bound.t()

    def check_forward(self, h, x=None, w=None):
        loss, lse = [torch.full((self.m,), float("nan"), device=DEV) for _ in range(2)]
        h.sgemm_cube_cross_entropy(self.x if x is None else x, self.w if w is None else w, self.targets, loss, bias=self.bias, lse=lse,
                                   weight_layout=self.layout)
        self.check_loss(loss, lse)
        return loss, lse

    def check_loss(self, loss, lse):
        assert bool(((lse.double() - self.lse).abs() <= self.lse_bound).all())
        # (infinite where the target itself is masked, on both sides)
        assert bool(((loss.double() == self.loss) | ((loss.double() - self.loss).abs() <= self.loss_bound)).all())
        assert bool((loss[self.targets < 0] == 0).all())

    def check_backward(self, h, x=None, w=None):
        nan = float("nan")
        dx, dw, db = torch.full_like(self.x, nan), torch.full_like(self.w, nan), torch.full((self.n,), nan, device=DEV)
        loss, lse = torch.full((self.m,), nan, device=DEV), torch.full((self.m,), nan, device=DEV)
        h.sgemm_cube_cross_entropy_backward(self.x if x is None else x, self.w if w is None else w, self.targets, self.dloss, dX=dx, dW=dw,
                                            dbias=db, bias=self.bias, loss=loss, lse=lse, weight_layout=self.layout)
        self.check_loss(loss, lse)
        for got, want, bound in ((dx, self.dx, self.dx_bound), (dw, self.dw, self.dw_bound), (db, self.db, self.db_bound)):
            assert bool(((got.double() - want).abs() <= bound).all())
            # and as a whole: a lost low word (2^-12) would show
            assert float((got.double() - want).norm()) <= 2.0 ** -16 * float(want.norm()) + 2.0 ** -16 * float(bound.norm())
        return dx, dw, db, loss, lse


# one row and one column; sizes on both sides of 64 columns, of tiles and of the forms for few rows; several waves of tiles
SIZES = [(1, 1, 1), (1, 5, 3), (2, 63, 8), (4, 65, 40), (7, 1000, 100), (33, 257, 64), (64, 513, 129), (129, 300, 70), (300, 1001, 257),
         (257, 8200, 65), (1100, 5000, 96)]


@pytest.mark.parametrize("layout", [WEIGHT_KN, WEIGHT_NK])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_forward(h, m, n, k, layout):
    c = Case(m, n, k, layout, bias=(m + n) % 2 == 1)
    loss, lse = c.check_forward(h)
    again = c.check_forward(h)
    assert torch.equal(loss, again[0]) and torch.equal(lse, again[1])
    packed = PackedMatrix(*c.w.shape)
    h.sgemm_cube_pack(c.w, packed)
    c.check_forward(h, w=packed)
    px = PackedMatrix(*c.x.shape)
    h.sgemm_cube_pack(c.x, px)
    c.check_forward(h, x=px, w=packed)


@pytest.mark.parametrize("layout", [WEIGHT_KN, WEIGHT_NK])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_backward(h, m, n, k, layout):
    c = Case(m, n, k, layout, bias=(m + n) % 2 == 0)
    first = c.check_backward(h)
    assert all(torch.equal(a, b) for a, b in zip(first, c.check_backward(h)))
    packed, px = PackedMatrix(*c.w.shape), PackedMatrix(*c.x.shape)
    h.sgemm_cube_pack(c.w, packed)
    h.sgemm_cube_pack(c.x, px)
    second = c.check_backward(h, x=px, w=packed)
    # (an FP32 X of up to 256 rows may take the linear layer's forms for few rows, which add in another order)
    assert m <= 256 or all(torch.equal(a, b) for a, b in zip(first, second))


# few rows, all of whose products read the weight as it is, packed or on odd addresses; long sums over the vocabulary
@pytest.mark.parametrize("layout", [WEIGHT_KN, WEIGHT_NK])
@pytest.mark.parametrize("m,n,k", [(1, 20000, 128), (2, 3001, 130), (4, 9999, 77), (6, 700, 1000), (9, 5003, 260), (16, 12001, 99), (17, 4000, 64),
                                   (40, 2050, 131), (150, 1500, 200)])
def test_gradients_of_few_rows(h, m, n, k, layout):
    c = Case(m, n, k, layout, seed=m)
    first = c.check_backward(h)
    assert all(torch.equal(a, b) for a, b in zip(first, c.check_backward(h)))
    packed = PackedMatrix(*c.w.shape)
    h.sgemm_cube_pack(c.w, packed)
    c.check_backward(h, w=packed)
    c.check_forward(h, w=packed)
    odd = strided(c.w, c.w.shape[1] + 5, 1)
    c.check_backward(h, w=odd)
    c.check_forward(h, w=odd)


@pytest.mark.parametrize("pair", [0, 1, 2])
@pytest.mark.parametrize("split", [0, 1])
def test_kernel_variants(pair, split):
    h = binding.Handle(0)
    h.sgemm_cube_set_option(binding.OPT_CTA_PAIR, pair)
    h.sgemm_cube_set_option(binding.OPT_SPLIT_K, split)
    for layout in (WEIGHT_KN, WEIGHT_NK):
        c = Case(390, 777, 1100, layout, seed=9)
        c.check_forward(h)
        c.check_backward(h)
    assert h.sgemm_cube_check()[0] == 0
    h.destroy()


@pytest.mark.parametrize("layout", [WEIGHT_KN, WEIGHT_NK])
def test_more_rows_than_a_piece(h, layout):
    """2400 rows of 190 000 logits are 1.8 GB: two pieces, whose weight gradients are added."""
    c = Case(2400, 190_000, 16, layout, seed=20, scale=1.0)
    c.check_backward(h)


@pytest.mark.parametrize("which", ["dx", "dw", "db", "dx dw", "none"])
def test_single_gradients(h, which):
    c = Case(70, 200, 33, WEIGHT_NK, seed=30)
    dx, dw, db, loss, lse = c.check_backward(h)
    out = dict(dX=torch.empty_like(dx) if "dx" in which else None, dW=torch.empty_like(dw) if "dw" in which else None,
               dbias=torch.empty_like(db) if "db" in which else None)
    h.sgemm_cube_cross_entropy_backward(c.x, c.w, c.targets, c.dloss, bias=c.bias, weight_layout=WEIGHT_NK, **out)
    for got, want in ((out["dX"], dx), (out["dW"], dw), (out["dbias"], db)):
        assert got is None or torch.equal(got, want)
    only = torch.empty_like(loss)
    h.sgemm_cube_cross_entropy_backward(c.x, c.w, c.targets, c.dloss, bias=c.bias, loss=only, weight_layout=WEIGHT_NK)
    assert bool(((only.double() - c.loss).abs() <= c.loss_bound).all())


def test_gradients_against_differences(h):
    c = Case(40, 90, 24, WEIGHT_NK, seed=40)
    dx, dw, db, _, _ = c.check_backward(h)

    def total(x, w, b):
        z = x @ w.t() + b
        known = c.targets >= 0
        loss = torch.logsumexp(z, 1) - z.gather(1, c.targets.clamp(min=0)[:, None])[:, 0]
        return float((torch.where(known, loss, 0.0) * c.dloss.double()).sum())

    args = [t.double() for t in (c.x, c.w, c.bias)]
    for i, grad in enumerate((dx, dw, db)):
        for s in range(3):
            step = rand(50 + s, *grad.shape).double()
            hi, lo = [list(args) for _ in range(2)]
            hi[i], lo[i] = args[i] + 1e-5 * step, args[i] - 1e-5 * step
            diff = (total(*hi) - total(*lo)) / 2e-5
            # third derivatives times 1e-10, and FP64's cancellation 1e-16 / 1e-5
            assert abs(diff - float((grad.double() * step).sum())) <= 1e-5 * float((grad.double() * step).abs().sum()) + 1e-9


def strided(t, ld, offset=0):
    buf = torch.full((t.shape[0] * ld + offset,), float("nan"), device=DEV)
    v = torch.as_strided(buf, t.shape, (ld, 1), offset)
    v.copy_(t)
    return v


@pytest.mark.parametrize("m", [3, 200])
def test_strides_and_any_alignment(h, m):
    c = Case(m, 150, 37, WEIGHT_KN, seed=60)
    x, w = strided(c.x, 41, 1), strided(c.w, 153, 3)
    c.check_forward(h, x=x, w=w)
    dx, dw = strided(torch.zeros_like(c.x), 39, 1), strided(torch.zeros_like(c.w), 155, 2)
    h.sgemm_cube_cross_entropy_backward(x, w, c.targets, c.dloss, dX=dx, dW=dw, bias=c.bias)
    assert bool(((dx.double() - c.dx).abs() <= c.dx_bound).all()) and bool(((dw.double() - c.dw).abs() <= c.dw_bound).all())


@pytest.mark.parametrize("m", [2, 150])
def test_masked_vocabulary_and_rows_with_nothing_left(h, m):
    c = Case(m, 400, 20, WEIGHT_NK, seed=70)
    c.bias[::3] = float("-inf")
    c.targets = (c.targets // 3 * 3 + 1).clamp_(max=399)
    c.targets64()
    c.dz = torch.nan_to_num(c.dz)
    c.check_forward(h)
    dx, db = torch.empty_like(c.x), torch.empty(400, device=DEV)
    h.sgemm_cube_cross_entropy_backward(c.x, c.w, c.targets, c.dloss, dX=dx, dbias=db, bias=c.bias, weight_layout=WEIGHT_NK)
    assert bool(((dx.double() - c.dx).abs() <= c.dx_bound).all()) and bool(((db.double() - c.db).abs() <= c.db_bound).all())
    # (399 is masked and a target: its column has -dloss; the other masked ones nothing)
    assert not db[:399:3].any()
    # a target that is masked: infinite loss, its row's gradient still p - 1[t]
    c.targets[0] = 3
    loss, lse = torch.empty(m, device=DEV), torch.empty(m, device=DEV)
    h.sgemm_cube_cross_entropy(c.x, c.w, c.targets, loss, bias=c.bias, lse=lse, weight_layout=WEIGHT_NK)
    assert float(loss[0]) == float("inf") and torch.equal(torch.isfinite(loss), (c.targets < 0) | (c.targets % 3 != 0))
    # nothing allowed at all
    c.bias.fill_(float("-inf"))
    c.targets[1] = -1
    dw = torch.empty_like(c.w)
    h.sgemm_cube_cross_entropy_backward(c.x, c.w, c.targets, c.dloss, dX=dx, dW=dw, dbias=db, bias=c.bias, loss=loss, lse=lse,
                                        weight_layout=WEIGHT_NK)
    assert bool((lse == float("-inf")).all()) and float(loss[0]) == float("inf") and float(loss[1]) == 0.0
    assert not dx.any() and not dw.any() and not db.any()


@pytest.mark.parametrize("m", [3, 140])
def test_targets_outside_the_vocabulary_and_nan(h, m):
    c = Case(m, 300, 16, WEIGHT_NK, seed=80)
    c.targets[:] = torch.arange(m, device=DEV) % 300
    c.targets[1] = 300
    c.targets[2] = -5
    loss, lse = torch.empty(m, device=DEV), torch.empty(m, device=DEV)
    dx = torch.empty_like(c.x)
    c.dloss[2] = float("nan")                                # of a row without target: not looked at
    h.sgemm_cube_cross_entropy_backward(c.x, c.w, c.targets, c.dloss, dX=dx, bias=c.bias, loss=loss, lse=lse, weight_layout=WEIGHT_NK)
    assert bool(torch.isnan(loss[1])) and float(loss[2]) == 0.0 and bool(torch.isfinite(lse).all())
    assert bool(torch.isnan(dx[1]).all()) and not dx[2].any() and bool(torch.isfinite(dx[3:]).all()) and bool(torch.isfinite(dx[0]).all())
    for bad in (float("nan"), float("inf")):
        x = c.x.clone()
        x[0, 3] = bad
        h.sgemm_cube_cross_entropy(x, c.w, c.targets, loss, bias=c.bias, lse=lse, weight_layout=WEIGHT_NK)
        assert bool(torch.isnan(lse[0])) and bool(torch.isfinite(lse[1:]).all())


@pytest.mark.parametrize("m", [2, 130])
def test_far_logits(h, m):
    """Logits of 2^20 with differences of one: the difference is taken before it is scaled."""
    n = 200
    x, w = torch.ones(m, 1, device=DEV), (2.0 ** 20 + torch.arange(n, device=DEV) % 7).view(n, 1)
    t = torch.zeros(m, dtype=torch.int64, device=DEV)
    loss = torch.empty(m, device=DEV)
    h.sgemm_cube_cross_entropy(x, w, t, loss, weight_layout=WEIGHT_NK)
    want = torch.logsumexp(w[:, 0].double(), 0) - 2.0 ** 20
    # the weights need 21 bits, which the words have: nothing but the sum's 200 u
    assert bool(((loss.double() - want).abs() <= 204 * U * want).all())


def test_no_rows(h):
    none = torch.empty(0, 8, device=DEV)
    w, t, v = rand(90, 8, 30), torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV)
    dw, db = torch.ones(8, 30, device=DEV), torch.ones(30, device=DEV)
    h.sgemm_cube_cross_entropy(none, w, t, v)
    h.sgemm_cube_cross_entropy_backward(none, w, t, v, dX=torch.empty(0, 8, device=DEV), dW=dw, dbias=db)
    assert not dw.any() and not db.any()


def test_refusals(h):
    lib, m, n, k = binding.load(), 5, 24, 8
    x, w, b, v, t = rand(91, m, k), rand(92, k, n), rand(93, n), rand(94, m), torch.zeros(m, dtype=torch.int64, device=DEV)
    out = {name: torch.empty(s, device=DEV) for name, s in dict(loss=(m,), lse=(m,), dx=(m, k), dw=(k, n), db=(n,)).items()}
    p = {name: o.data_ptr() for name, o in out.items()}
    ox, ow = binding._Operand(x.data_ptr(), k, None, None, 0, None), binding._Operand(w.data_ptr(), n, None, None, 0, None)
    short = binding._Operand(w.data_ptr(), n - 1, None, None, 0, None)
    packed = PackedMatrix(k, n)
    h.sgemm_cube_pack(w, packed)
    o = packed.operand
    odd = binding._Operand(None, 0, o.hi_dev + 2, o.lo_dev, o.ld16, o.exp_dev)

    def fwd(m=m, n=n, k=k, x=ox, w=ow, layout=0, b=b.data_ptr(), t=t.data_ptr(), loss=p["loss"], lse=p["lse"]):
        return lib.sgemm_cube_cross_entropy(h._h, m, n, k, x, w, layout, b, t, loss, lse, None)

    def bwd(m=m, n=n, k=k, x=ox, w=ow, layout=0, b=b.data_ptr(), t=t.data_ptr(), loss=p["loss"], lse=p["lse"], d=v.data_ptr(), dx=p["dx"],
            lddx=k, dw=p["dw"], lddw=n, db=p["db"]):
        return lib.sgemm_cube_cross_entropy_backward(h._h, m, n, k, x, w, layout, b, t, d, loss, lse, dx, lddx, dw, lddw, db, None)

    assert fwd() == 0 and bwd() == 0 and fwd(loss=None) == 0 and fwd(lse=None) == 0
    before = h.sgemm_cube_launch_count()
    for bad in (dict(m=-1), dict(n=0), dict(k=0), dict(n=2 ** 31 - 1), dict(layout=2), dict(x=None), dict(w=None), dict(w=short), dict(t=None),
                dict(t=t.data_ptr() + 4), dict(b=b.data_ptr() + 2), dict(loss=p["loss"] + 1), dict(lse=p["lse"] + 2)):
        assert fwd(**bad) == INVALID_ARG, bad
        assert bwd(**bad) == INVALID_ARG, bad
    assert fwd(w=odd) == MISALIGNED and bwd(w=odd) == MISALIGNED
    assert fwd(loss=None, lse=None) == INVALID_ARG
    for bad in (dict(d=None), dict(d=v.data_ptr() + 1), dict(dx=p["dx"] + 2), dict(dw=p["dw"] + 2), dict(db=p["db"] + 2), dict(lddx=k - 1),
                dict(lddw=n - 1)):
        assert bwd(**bad) == INVALID_ARG, bad
    assert h.sgemm_cube_launch_count() == before
