"""Distillation over the values that logits and teachers can hold: finite masks,
magnitudes whose quotient by the temperature is large, small temperatures.

Tolerances as in test_gpu_rows.py.  They hold for any finite logits: an exponent
(s - max) / T passes five roundings (the difference, log2(e), its quotient by T,
the product, log q) and the loss four more, nine units against the twelve of
check_distill.  The temperatures are powers of two or small integers, without a
rounding of their own, and the teachers' entries share their mass evenly or
leave it to one of them, so that p adds no error that scales with the logits.
The widths are rows of one pack a thread, of several, and rows too long for
registers.
"""
import math

import pytest
import torch

import paper_2608_09713_amd as sp
from tests.test_gpu_rows import DEV, DTYPES, check_distill, gen, normal

pytestmark = pytest.mark.gpu

WIDTHS = [60, 5000, 20003, 140001]


@pytest.fixture(scope="module", autouse=True)
def _library():
    sp.library()


def check_both(s, vals, cols, T, what):
    """Loss alone and with the gradient against the definition; a row of weight 0 has a finite loss too."""
    m = s.shape[0]
    w = torch.linspace(0.25, 1.5, m)
    w[::5] = 0.0
    S, teacher = s.to(DEV), (vals.to(DEV), cols.to(DEV))
    loss, grad = sp.distill_grad(S, teacher, T, w.to(DEV))
    assert bool(loss.isfinite().all()) and bool(grad.isfinite().all()), (what, T)
    assert torch.equal(sp.distill(S, teacher, T), loss), (what, T)
    check_distill(s, [(cols[r], vals[r]) for r in range(m)], T, w, loss.cpu(), grad.cpu(), (what, T))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("v", WIDTHS)
def test_finite_masks(dtype, v):
    """Rows masked by a finite value at their start, in scattered packs, at their end and whole."""
    g = gen(v + 1)
    masks = [torch.finfo(dtype).min] + ([-6e4, -3e4] if dtype == torch.float16 else [-1e30, -1e20, -1e10, -1e9])
    n = 16 // (torch.finfo(dtype).bits // 8)
    rows, cols = [], []
    for mask in masks:
        for where in ("start", "packs", "end", "whole"):
            hidden = torch.zeros(v, dtype=torch.bool)
            if where == "start":
                hidden[: v // 2 + 3] = True
            elif where == "packs":
                hidden = (torch.rand(v // n + 1, generator=g) < 0.4).repeat_interleave(n)[:v]
            elif where == "end":
                hidden[v // 3:] = True
            else:
                hidden[:] = True
            s = normal((v,), dtype, g, 2.0)
            s[hidden] = mask
            shown = torch.arange(v) if where == "whole" else (~hidden).nonzero()[:, 0]
            rows.append(s)
            cols.append(torch.cat([shown[torch.randperm(shown.numel(), generator=g)[:6]], hidden.nonzero()[:1, 0]]))
    s, cols = torch.stack(rows), torch.stack(cols)
    vals = torch.zeros((len(rows), 7))
    vals[:, 6] = -math.inf  # (no mass at the masked one)
    for T in (0.25, 1.0, 2.0, 3.0, 4.0):
        check_both(s, vals, cols, T, "masks")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", WIDTHS)
def test_large_magnitudes(dtype, v):
    """Rows of one large value, rows with several columns at it, and rows of
    values around it, of both signs."""
    g = gen(v + 2)
    rows, cols, vals = [], [], []
    for k in range(5, 30, 2):
        for sign in (1.0, -1.0):
            for kind in ("same", "ties", "around"):
                at = torch.randperm(v, generator=g)[:5]
                s = torch.full((v,), sign * 10.0 ** k)
                if kind == "ties":
                    s = normal((v,), torch.float32, g, 2.0) if sign > 0 else s * (1.0 + torch.rand(v, generator=g))
                    s[at] = sign * 10.0 ** k
                elif kind == "around":
                    s *= 1.0 + torch.rand(v, generator=g)
                rows.append(s.to(dtype))
                cols.append(at)
                vals.append([0.0] + [-math.inf if kind == "around" else 0.0] * 4)
    s, cols, vals = torch.stack(rows), torch.stack(cols), torch.tensor(vals)
    for T in (0.125, 1.0):
        check_both(s, vals, cols, T, "magnitudes")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("v", WIDTHS)
def test_small_temperatures(dtype, v):
    g = gen(v + 3)
    s = normal((7, v), dtype, g, 5.0)
    cols = torch.stack([torch.randperm(v, generator=g)[:9] for _ in range(7)])
    vals = torch.stack([torch.randperm(9, generator=g) for _ in range(7)]).float()
    cols[2, 0], vals[2, 0] = s[2].float().argmax(), 20.0
    for T in (2.0 ** -10, 2.0 ** -20, 2.0 ** -30):
        check_both(s, vals, cols, T, "small temperature")


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_columns(dtype):
    """Rows of no columns have nothing to match, with and without entries."""
    S = torch.zeros((5, 0), dtype=dtype, device=DEV)

    def rows(lens):
        rp = torch.tensor([0] + lens, device=DEV).cumsum(0)
        nnz = sum(lens)
        return sp.DeviceCSR(5, 0, rp, torch.zeros(nnz, dtype=torch.int32, device=DEV),
                            torch.ones(nnz, device=DEV), nnz)

    def pair(k):
        return torch.ones((5, k), device=DEV), torch.zeros((5, k), dtype=torch.int64, device=DEV)

    for teacher in (pair(0), pair(1), pair(300), rows([0] * 5), rows([0, 1, 0, 0, 0]), rows([9] * 5)):
        loss = sp.distill(S, teacher)
        assert loss.shape == (5,) and not loss.any()
        loss, grad = sp.distill_grad(S, teacher, 2.0, torch.ones(5, device=DEV))
        assert loss.shape == (5,) and not loss.any() and grad.shape == (5, 0) and grad.dtype == dtype


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("v", WIDTHS)
def test_order_of_two_listings(dtype, v):
    """A column listed twice in a row: the gradient has the same bits whichever
    listing comes first, near each other or in different wavefronts' entries.

    With log2(e) / T = 1 and whole teacher values the row's exponentials are
    powers of two and their sum is exact, so that p itself has no order."""
    g = gen(v + 4)
    m, k, twice = 400, 100, 30
    T = float(torch.tensor(1.4426950408889634))
    s = normal((m, v), dtype, g, 2.0)
    one = torch.rand((m, k - twice), generator=g).mul_(v).long().clamp_(max=v - 1)
    cols = torch.cat([one, one[:, :twice]], 1)
    vals = torch.randint(-9, 1, (m, k), generator=g).float()
    other = torch.arange(k)
    other[:twice], other[k - twice:] = torch.arange(k - twice, k), torch.arange(twice)
    S = s.to(DEV)
    loss, grad = sp.distill_grad(S, (vals.to(DEV), cols.to(DEV)), T)
    # the two listings' values change places
    swapped = sp.distill_grad(S, (vals[:, other].to(DEV), cols.to(DEV)), T)
    assert bool((cols[:, other] == cols).all())
    # columns that are listed three times or more have no such promise
    count = torch.zeros((m, v)).scatter_add_(1, cols, torch.ones((m, k)))
    kept = (count < 3).to(DEV)
    assert int((count == 2).sum()) > 100
    assert torch.equal(grad[kept], swapped[1][kept])
    for _ in range(3):
        again = sp.distill_grad(S, (vals.to(DEV), cols.to(DEV)), T)
        assert torch.equal(again[0], loss) and torch.equal(again[1][kept], grad[kept])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("v", WIDTHS)
def test_columns_listed_often(dtype, v):
    """Rows filled up with one column, without mass or with it, and rows of few columns in turn."""
    g = gen(v + 5)
    k = 200
    s = normal((4, v), dtype, g, 2.0)
    cols = torch.stack([torch.randperm(v, generator=g)[:50].repeat(4) for _ in range(4)])
    vals = normal((4, k), torch.float32, g)
    cols[0, 20:], vals[0, 20:] = 0, -math.inf
    cols[1, 20:] = 0
    cols[2] = torch.arange(k) % 5
    cols[3] = torch.arange(k) // 40
    check_both(s, vals, cols, 1.0, "listed often")


@pytest.mark.parametrize("dtype", DTYPES)
def test_one_column_of_a_wider_tensor(dtype):
    """Rows of one element are contiguous whatever the stride between columns."""
    g = gen(7)
    wide = normal((6, 12), dtype, g).to(DEV)
    x, same = wide[:, 3::9], wide[:, 3:4].contiguous()
    assert x.shape == (6, 1) and x.stride(1) != 1
    tok = torch.tensor([5, 0, -1, 3], device=DEV)
    assert torch.equal(sp.embed(tok, x, 2.0), sp.embed(tok, same, 2.0))
    assert torch.equal(sp.embed_grad(tok, x[:4], 9), sp.embed_grad(tok, same[:4], 9))
    for got, want in zip(sp.layer_norm(x), sp.layer_norm(same)):
        assert torch.equal(got, want)
    S = normal((6, 40), dtype, g).to(DEV)
    cols = torch.randint(0, 40, (6, 12), generator=g).to(DEV)
    got = sp.distill_grad(S, (x, cols[:, 3::9]))
    want = sp.distill_grad(S, (same, cols[:, 3:4].contiguous()))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
