"""Rows that are sure of their target: loss and gradient keep their digits however
near the target's probability is to 1.

One logit a at the target and zeros elsewhere: loss = log1p((V - 1) e^-a), which is
-a + log(V - 1 + e^a) where a is below 0.  Tolerances, fixed from the arithmetic (u =
2^-24): the logits are exact, and so is the sum of V - 1 ones; e^-a has its exponent's
two roundings (by log2(e) and the product: 2 |a| u) and the function's (2 u), which
the product with V - 1 and the logarithm (8 u together) pass on: e = (2 |a| + 12) u of
the loss.  The target's entry of G adds the exponential's 8 u, and dx and dW (one term
that is not 0) 4 u and the roundings of G and of the result to the type.  In IEEE
16-bit floats G loses at most 2^-25 of its unit, 2^-14 of the largest weight.
"""
import math

import pytest
import torch

import paper_2608_09713_amd as sp
from tests.test_gpu_rows import DEV, DTYPES, ROUND, TINY, U, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    sp.library()


def problem(N, V, dtype):
    """(x, w, targets, a): a from -6 to 40, targets over all columns, the last one among them."""
    a = (torch.arange(N) * 7 % 93).float() / 2 - 6.0  # (multiples of 1/2: exact in every type)
    t = V - 1 - torch.arange(N) * 5 % V
    x = torch.zeros((N, V))
    x[torch.arange(N), t] = a
    return x.to(dtype), torch.eye(V).to(dtype), t, a.double()


def want(a, V):
    loss = torch.log1p((V - 1) * torch.exp(-a))
    return loss, a + loss


# (few rows by one reading of W, and tiles; a target alone in its piece: 65, 129 and 257 columns)
SIZES = [(5, 16), (41, 300), (16, 65), (9, 1), (130, 300), (300, 129), (300, 257), (1100, 600)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,V", SIZES)
def test_loss(dtype, N, V):
    x, w, t, a = problem(N, V, dtype)
    loss, lse = want(a, V)
    got, got_lse = sp.linear_cross_entropy(x.to(DEV), w.to(DEV), t.to(DEV))
    e = (2 * a.abs() + 12) * U
    check(got, loss, e * loss, "loss")
    # (of log(V - 1 + e^a) as a sum: the loss's, and a rounding of the sum)
    check(got_lse, lse, e * loss + U * lse.abs(), "lse")
    t[::3] = -1  # (padding: the sum takes all columns)
    got, got_lse = sp.linear_cross_entropy(x.to(DEV), w.to(DEV), t.to(DEV))
    check(got, torch.where(t < 0, 0.0, loss), torch.where(t < 0, 0.0, e * loss), "loss beside padding")
    check(got_lse, lse, (2 * a.abs() + 12 + V) * U * (1 + loss.abs()) + U * lse.abs(), "lse of padding")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,V", SIZES)
def test_gradient(dtype, N, V):
    x, w, t, a = problem(N, V, dtype)
    loss, _ = want(a, V)
    got, dx, _ = sp.linear_cross_entropy_grad(x.to(DEV), w.to(DEV), t.to(DEV))
    e = (2 * a.abs() + 12) * U
    check(got, loss, e * loss, "loss")
    g = torch.expm1(-loss)
    r = ROUND[dtype]
    lost = 2.0 ** -38 if dtype == torch.float16 else 0.0
    # (d expm1(-l) = -e^-l dl: at most the loss's relative error of g)
    tol = (e + 12 * U + 2.01 * r) * g.abs() + lost + TINY[dtype]
    check(dx[torch.arange(N), t], g, tol, "dx at the target")
    # the row's entries add up to 0: the target's is the others' sum
    if dtype == torch.float32:
        rest = dx.double().sum(1).cpu()
        assert (rest.abs() <= (4 * a.abs() + 40) * U * 2 * g.abs() + V * TINY[dtype]).all()


def test_values_of_infinite_logits():
    def loss(column, t):
        got = sp.linear_cross_entropy(torch.ones((1, 1), device=DEV), torch.tensor(column, device=DEV)[:, None],
                                      torch.tensor([t], device=DEV))
        return float(got[0]), float(got[1])

    inf = math.inf
    assert all(map(math.isnan, loss([inf, 0.0], 0)))          # inf - inf
    assert not math.isfinite(loss([inf, 0.0], 1)[0])
    assert loss([-inf, 0.0], 0) == (inf, 0.0)                 # (a target of no probability)
    assert loss([-inf, 0.0], 1) == (0.0, 0.0)                 # (-inf elsewhere adds nothing)
    assert all(map(math.isnan, loss([math.nan, 0.0], 0))) and all(map(math.isnan, loss([math.nan, 0.0], 1)))
    assert loss([5.0], 0) == (0.0, 5.0)
