"""Cross entropy of a linear layer on the GPU against a plain 64-bit form.

Tolerances, fixed from the arithmetic: with u = 2^-24 and r the rounding of the
inputs' type (2^-24, 2^-11, 2^-8),
- a logit is a sum of d products, exact for 16-bit types: off by at most ez =
  (d + 4) u times the sum of its terms' magnitudes (the multiplications by scale
  and log2(e), and that of the product in 32 bits, are the rest), and by 2 u of
  itself where a base is subtracted;
- the exponentials' sum has terms of relative error 2 u (the function) + what
  their exponents are off by; V terms are added within tiles by 32 in a lane, 8
  steps and then over at most 64 tiles a lane: K = 256 covers them; lse is off by
  that, and loss by both logits;
- an entry of G has the relative error of its exponents, and two roundings (the
  exponential's, its own); the target's one.  The division by the largest weight
  and the multiplication by it add 2 u.  Sums over v (rows) add (V + 4) u ((N + 4)
  u) of their magnitudes.  In IEEE 16-bit floats an entry also loses at
  most 2^-25 of the unit, which is 2^-14 of the largest weight, and an
  exponential 2^-40 of its row's largest.
"""
import pytest
import torch

import paper_2608_09713_amd as sp
from tests import training_reference as ref
from tests.test_gpu_rows import DEV, DTYPES, ROUND, TINY, U, check, gen, normal

pytestmark = pytest.mark.gpu
K = 256
LOG2E = 1.4426950408889634


@pytest.fixture(scope="module", autouse=True)
def _library():
    sp.library()


def problem(N, V, D, dtype, seed=0, spread=2.0, padding=True, weights=True):
    g = gen(1000 * seed + N + V + D)
    w = normal((V, D), dtype, g, spread / D ** 0.5)
    t = torch.randint(0, V, (N,), generator=g)
    x = (torch.randn((N, D), generator=g) + w[t].float() * torch.rand((N, 1), generator=g) * 4.0).to(dtype)
    if padding and N > 2:
        t[torch.rand(N, generator=g) < 0.2] = -1
        t[0], t[1] = V, 1 << 40
    wt = None
    if weights:
        wt = torch.rand(N, generator=g) * 2 - 0.5
        if N > 4:
            wt[torch.rand(N, generator=g) < 0.2] = 0.0
    return x, w, t, wt


def errors(want, V, D):
    """(of a logit, of lse, of loss) per row."""
    ez = (D + 4) * U * want["zmag"]
    big = want["lse"].abs() + want["hit"].abs()
    e_lse = 2 * ez + K * U + 4 * U * big
    return ez, e_lse, e_lse + 2 * ez + 4 * U * big


def check_loss(got, want, V, D):
    ez, e_lse, e_loss = errors(want, V, D)
    check(got[0], want["loss"], torch.where(want["named"], e_loss, 0.0) + TINY[torch.float32], "loss")
    if len(got) > 1:
        check(got[1], want["lse"], e_lse + TINY[torch.float32], "lse")


def check_grad(dx, dw, want, wt, N, V, D, dtype):
    ez, e_lse, _ = errors(want, V, D)
    r = ROUND[dtype]
    rel = ((ez + e_lse) * 2 + 10 * U + 4 * U * (want["lse"].abs() + want["zmag"])).max()
    lost = 0.0
    if dtype == torch.float16:
        lost = 2.0 ** -38 * float(wt.abs().max())
    tol_dx = (r * 1.01 + rel + (V + 4) * U) * want["dx_mag"] + (r * 1.01 + rel) * want["q_dx"] + lost * want["w_abs"]
    tol_dw = (r * 1.01 + rel + (N + 4) * U) * want["dw_mag"] + (r * 1.01 + rel) * want["q_dw"] + lost * want["x_abs"]
    check(dx, want["dx"], tol_dx + r * (want["dx"].abs() + tol_dx) + TINY[dtype], "dx")
    check(dw, want["dw"], tol_dw + r * (want["dw"].abs() + tol_dw) + TINY[dtype], "dw")
    unused = ~want["used"]
    assert not dx.reshape(N, D).cpu()[unused].any()


SIZES = [(1, 1, 1), (2, 7, 5), (1, 5000, 72), (3, 300, 8), (17, 64, 64), (130, 300, 64), (64, 20000, 64),
         (257, 515, 100), (300, 129, 256), (65, 1025, 1001), (1600, 8191, 24)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,V,D", SIZES)
def test_loss(dtype, N, V, D):
    x, w, t, _ = problem(N, V, D, dtype)
    for scale in (1.0, -0.375):
        want = ref.cross_entropy(x.double(), w.double(), t, scale)
        got = sp.linear_cross_entropy(x.to(DEV), w.to(DEV), t.to(DEV), scale)
        check_loss(got, want, V, D)
        again = sp.linear_cross_entropy(x.to(DEV), w.to(DEV), t.to(DEV), scale)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,V,D", SIZES)
def test_gradient(dtype, N, V, D):
    x, w, t, wt = problem(N, V, D, dtype)
    for scale, weights in ((1.0, wt), (0.5, None)):
        one = torch.ones(N) if weights is None else weights
        want = ref.cross_entropy(x.double(), w.double(), t, scale, one.double())
        args = (x.to(DEV), w.to(DEV), t.to(DEV), scale, None if weights is None else weights.to(DEV))
        loss, dx, dw = sp.linear_cross_entropy_grad(*args)
        check_loss((loss,), want, V, D)
        check_grad(dx, dw, want, one, N, V, D, dtype)
        again = sp.linear_cross_entropy_grad(*args)
        assert torch.equal(dx, again[1]) and torch.equal(dw, again[2])


def test_gradient_against_differences():
    # in 32 bits: differences of the 64-bit loss along two directions
    x, w, t, wt = problem(40, 90, 24, torch.float32)
    _, dx, dw = sp.linear_cross_entropy_grad(x.to(DEV), w.to(DEV), t.to(DEV), 0.7, wt.to(DEV))
    g = gen(5)
    ux, uw = torch.randn(x.shape, generator=g).double(), torch.randn(w.shape, generator=g).double()

    def loss(h):
        return float((ref.cross_entropy(x.double() + h * ux, w.double() + h * uw, t, 0.7)["loss"] * wt.double()).sum())

    h = 1e-5
    slope = (loss(h) - loss(-h)) / (2 * h)
    got = float((dx.cpu().double() * ux).sum() + (dw.cpu().double() * uw).sum())
    # (the difference itself: h^2 times third derivatives, and 1e-16 / h of the losses' sum)
    assert abs(got - slope) <= 1e-5 * (dx.abs().cpu().double() * ux.abs()).sum() + 1e-5 * (dw.abs().cpu().double() * uw.abs()).sum()


# (few rows by tiles: many columns in whole steps; beside them, by one reading of W)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,V,D", [(17, 25000, 64), (33, 25000, 64), (64, 24577, 128), (64, 24577, 130), (64, 20000, 64)])
def test_few_rows_of_many_columns(dtype, N, V, D):
    x, w, t, _ = problem(N, V, D, dtype)
    want = ref.cross_entropy(x.double(), w.double(), t, 1.0)
    check_loss(sp.linear_cross_entropy(x.to(DEV), w.to(DEV), t.to(DEV)), want, V, D)


# (tiles of 128 x 128, others than the ones above: of the logits, of both products of
# which dX's is split, and of dX's whole; rows that are whole steps, and odd ones)
@pytest.mark.parametrize("N,V,D", [(128, 32700, 33), (130, 32760, 64), (300, 9000, 128), (300, 9000, 129),
                                   (4090, 40, 2045), (4096, 50, 2048)])
def test_larger_tiles_of_32_bits(N, V, D):
    x, w, t, wt = problem(N, V, D, torch.float32)
    want = ref.cross_entropy(x.double(), w.double(), t, 1.0, wt.double())
    loss, dx, dw = sp.linear_cross_entropy_grad(x.to(DEV), w.to(DEV), t.to(DEV), 1.0, wt.to(DEV))
    check_loss((loss,), want, V, D)
    check_grad(dx, dw, want, wt, N, V, D, torch.float32)
    assert torch.equal(sp.linear_cross_entropy(x.to(DEV), w.to(DEV), t.to(DEV))[0], loss)


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_and_leading_dimensions(dtype):
    N, V, D = 36, 77, 64
    x, w, t, wt = problem(N, V, D, dtype)
    want = sp.linear_cross_entropy(x.to(DEV), w.to(DEV), t.to(DEV))
    grads = sp.linear_cross_entropy_grad(x.to(DEV), w.to(DEV), t.to(DEV), 1.0, wt.to(DEV))
    wide_x, wide_w = torch.zeros((N, D + 5), dtype=dtype, device=DEV), torch.zeros((V, D + 8), dtype=dtype, device=DEV)
    wide_x[:, 3:3 + D], wide_w[:, 8:] = x.to(DEV), w.to(DEV)
    t2 = torch.stack([t, t], 1).to(DEV)[:, 0]
    got = sp.linear_cross_entropy(wide_x[:, 3:3 + D], wide_w[:, 8:], t2)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    got = sp.linear_cross_entropy_grad(wide_x[:, 3:3 + D], wide_w[:, 8:], t2, 1.0, wt.to(DEV))
    assert all(torch.equal(a, b) for a, b in zip(got, grads))
    x3 = x.to(DEV).view(4, 9, D)
    loss, lse = sp.linear_cross_entropy(x3, w.to(DEV), t.clamp(-1, V).int().to(DEV).view(4, 9))
    assert loss.shape == (4, 9) and torch.equal(loss.view(-1), want[0]) and torch.equal(lse.view(-1), want[1])
    loss, dx, dw = sp.linear_cross_entropy_grad(x3, w.to(DEV), t.to(DEV).view(4, 9), 1.0, wt.to(DEV).view(4, 9))
    assert dx.shape == x3.shape and torch.equal(dx.view(N, D), grads[1]) and torch.equal(dw, grads[2])


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_that_take_no_part(dtype):
    # what stands in padding and in rows of weight 0 reaches nothing
    N, V, D = 50, 200, 40
    x, w, t, wt = problem(N, V, D, dtype, padding=False)
    t[::3] = -1
    wt[1::3] = 0.0
    clean = sp.linear_cross_entropy_grad(x.to(DEV), w.to(DEV), t.to(DEV), 1.0, wt.to(DEV))
    bad = x.clone()
    bad[::3] = float("nan")
    bad[1::3] = float("inf")
    got = sp.linear_cross_entropy_grad(bad.to(DEV), w.to(DEV), t.to(DEV), 1.0, wt.to(DEV))
    assert not got[0][::3].any() and torch.equal(got[0][2::3], clean[0][2::3])
    assert torch.equal(got[1], clean[1]) and torch.equal(got[2], clean[2])
    assert not got[1][::3].any() and not got[1][1::3].any()
    loss, _ = sp.linear_cross_entropy(bad.to(DEV), w.to(DEV), t.to(DEV))
    assert not loss[::3].any()
    none = sp.linear_cross_entropy_grad(bad.to(DEV), w.to(DEV), torch.full_like(t, -1).to(DEV))
    assert not any(bool(a.any()) for a in none)


def test_no_rows():
    w = torch.randn((30, 12), device=DEV)
    x, t = torch.empty((0, 12), device=DEV), torch.empty(0, dtype=torch.int64, device=DEV)
    loss, lse = sp.linear_cross_entropy(x, w, t)
    assert loss.shape == lse.shape == (0,)
    loss, dx, dw = sp.linear_cross_entropy_grad(x, w, t)
    assert dx.shape == (0, 12) and dw.shape == w.shape and not dw.any()


def test_large_and_infinite_logits():
    # logits of +-1e4 and more, a row that is sure of its target, one that is sure of another
    D = 8
    w = torch.eye(8)
    x = torch.zeros((6, D))
    x[0] = torch.tensor([3e4, -3e4, 0, 0, 0, 0, 0, 0])
    x[1] = x[0]
    x[2, 3] = 60.0
    x[3] = 1e30
    x[4, 0], x[4, 1:] = 3e38, -3e38
    x[5, 2] = float("nan")
    t = torch.tensor([0, 1, 3, 5, 0, 1])
    loss, dx, dw = sp.linear_cross_entropy_grad(x.to(DEV), w.to(DEV), t.to(DEV), 1.0,
                                                torch.tensor([1., 1, 1, 1, 1, 0]).to(DEV))
    loss = loss.cpu().double()
    assert loss[0] == 0 and abs(loss[1] - 6e4) <= 6e4 * 8 * U and loss[4] == 0 and torch.isnan(loss[5])
    assert abs(loss[2] - 7 * 8.75651076e-27) <= 60 * 8 * U
    assert abs(loss[3] - 2.0794415) < 1e30 * 8 * U
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all()
    want = torch.zeros(8)
    want[0], want[1] = 1.0, -1.0
    assert torch.equal(dx[1].cpu(), want) and not dx[0].any()
    inf = sp.linear_cross_entropy(torch.tensor([[1.0, 1.0]]).to(DEV),
                                  torch.tensor([[3e38, 3e38], [1.0, 0.0]]).to(DEV), torch.tensor([1]).to(DEV))
    assert not torch.isfinite(inf[0]).any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_sure_rows_keep_their_gradient(dtype):
    # 1 - q far below the type's step: the gradient is that of the 32-bit logits
    D = 16
    w = torch.eye(D).to(dtype)
    x = torch.zeros((4, D), dtype=dtype)
    for k, z in enumerate((8.0, 16.0, 24.0, 32.0)):
        x[k, k] = z
    t = torch.arange(4)
    want = ref.cross_entropy(x.double(), w.double(), t, 1.0, torch.ones(4, dtype=torch.float64))
    _, dx, dw = sp.linear_cross_entropy_grad(x.to(DEV), w.to(DEV), t.to(DEV))
    check_grad(dx, dw, want, torch.ones(4), 4, D, D, dtype)
    assert float(dx[1, 1]) < 0 and float(dx[0, 0]) < float(dx[1, 1])


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_in_several_turns(dtype):
    # more rows than are taken at a time (2^17): dW is added up over the turns
    N, V, D, period = (1 << 17) + 300, 3, 8, 307
    x, w, t, wt = problem(period, V, D, dtype)
    index = torch.arange(N) % period
    want = ref.cross_entropy(x.double(), w.double(), t, 1.0, wt.double())
    loss, dx, dw = sp.linear_cross_entropy_grad(x[index].to(DEV), w.to(DEV), t[index].to(DEV), 1.0, wt[index].to(DEV))
    small = sp.linear_cross_entropy_grad(x.to(DEV), w.to(DEV), t.to(DEV), 1.0, wt.to(DEV))
    check_grad(small[1], small[2], want, wt, period, V, D, dtype)
    assert torch.equal(loss, small[0][index.to(DEV)]) and torch.equal(dx, small[1][index.to(DEV)])
    full = ref.cross_entropy(x[index].double(), w.double(), t[index], 1.0, wt[index].double())
    check_grad(dx, dw, full, wt, N, V, D, dtype)


def test_loss_in_several_turns():
    N, V, D, period = (1 << 19) + 77, 8192, 8, 1531
    x, w, t, _ = problem(period, V, D, torch.bfloat16)
    index = (torch.arange(N) % period).to(DEV)
    x, w, t = x.to(DEV), w.to(DEV), t.to(DEV)
    small = sp.linear_cross_entropy(x, w, t)
    loss, lse = sp.linear_cross_entropy(x[index], w, t[index])
    # (tiles of another size have sums in another order)
    bound = K * U + 8 * U * small[1].abs()
    assert ((lse - small[1][index]).abs() <= bound[index]).all()
    assert ((loss - small[0][index]).abs() <= 2 * bound[index] * (t[index] >= 0)).all()
    assert torch.equal(lse[period:2 * period], lse[:period])
