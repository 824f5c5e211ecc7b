"""Lookup, layer norm and distillation on the GPU against plain 64-bit forms.

Tolerances, fixed from the arithmetic: with u = 2^-24 (32-bit floats) and r the
rounding of the output type (2^-24, 2^-11, 2^-8),
- a lookup of one token is one product, so its bits are given;
- a sum of n terms is off by at most (n + 3) u times the sum of the terms'
  magnitudes, then r of the result;
- a row's mean and variance are sums of at most 96 terms per thread and a tree
  of 10 levels: K = 128 covers them with the few operations that follow;
- z = (s - max) / T is off by 4 u |z|, which the exponential passes on as a
  relative error; the sums behind L as above.
"""
import math

import pytest
import torch

import paper_2608_09713_amd as sp
from tests import rows_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}
DTYPES = [torch.float32, torch.float16, torch.bfloat16]
K = 128


@pytest.fixture(scope="module", autouse=True)
def _library():
    sp.library()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(shape, dtype, g, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def check(got, want, tol, what):
    got = ref.f64(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    err = (got - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / tol)[bad].max())} times"


def csr(g, m, n, most, dtype=torch.float32, values=True, long_row=None):
    """Random CSR with empty rows; long_row: a row that holds that many entries
    (columns may repeat there)."""
    lens = torch.randint(0, most + 1, (m,), generator=g)
    lens[torch.rand(m, generator=g) < 0.2] = 0
    if long_row:
        lens[m // 2] = long_row
    rp = torch.zeros(m + 1, dtype=torch.int64)
    rp[1:] = lens.cumsum(0)
    nnz = int(rp[-1])
    cols = torch.randint(0, n, (nnz,), generator=g)
    vals = normal((nnz,), dtype, g) if values else None
    rows = torch.repeat_interleave(torch.arange(m), lens)
    A = sp.DeviceCSR(m, n, rp.to(DEV), cols.int().to(DEV), None if vals is None else vals.to(DEV), nnz)
    return A, rows, cols, torch.ones(nnz, dtype=torch.float64) if vals is None else vals.double()


def sums_tol(count, mag, want, dtype):
    return (count + 3) * U * mag + ROUND[dtype] * want.abs() + TINY[dtype]


# ---- lookup

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [1, 7, 8, 64, 65, 520, 1001, 2056, 5000])
@pytest.mark.parametrize("n", [1, 130])
def test_tokens(dtype, d, n):
    g = gen(d + n)
    v = 97
    W = normal((v, d), dtype, g).to(DEV)
    tok = torch.randint(0, v, (n,), generator=g)
    tok[torch.rand(n, generator=g) < 0.2] = -1
    if n > 3:
        tok[0], tok[1], tok[2] = v, v - 1, 1 << 40
    tok = tok.to(DEV)
    scale = math.sqrt(d)
    ok = (tok >= 0) & (tok < v)
    want = torch.where(ok[:, None], (W[tok.clamp(0, v - 1)].float() * scale).to(dtype), torch.zeros((), dtype=dtype, device=DEV))
    assert torch.equal(sp.embed(tok, W, scale), want)
    if n > 3:
        small = tok.clamp(-1, v).int()
        assert torch.equal(sp.embed(small.view(2, n // 2), W, scale), want.view(2, n // 2, d))
    # a slice of a wider table at an odd offset, strided tokens
    wide = torch.zeros((v, d + 5), dtype=dtype, device=DEV)
    wide[:, 3:3 + d] = W
    two = torch.stack([tok, tok.flip(0)], 1)
    assert torch.equal(sp.embed(two[:, 0], wide[:, 3:3 + d], scale), want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [1, 9, 64, 250, 1001, 4104])
@pytest.mark.parametrize("values", [True, False])
def test_csr_lookup(dtype, d, values):
    g = gen(d)
    m, n = 301, 113
    A, rows, cols, vals = csr(g, m, n, 30, values=values, long_row=3001)
    W = normal((n, d), dtype, g)
    want, mag = ref.lookup(rows, cols, vals, W.double(), m, 0.25)
    count = torch.bincount(rows, minlength=m)[:, None]
    got = sp.embed(A, W.to(DEV), 0.25)
    check(got, want, sums_tol(count, mag, want, dtype), "csr lookup")
    assert torch.equal(got, sp.embed(A, W.to(DEV), 0.25))


def token_sets(n, v, g):
    skew = (v * torch.rand(n, generator=g) ** 6).long().clamp_(0, v - 1)
    return {"uniform": torch.randint(0, v, (n,), generator=g), "skewed": skew,
            "one": torch.full((n,), v - 1), "padding": torch.full((n,), -1),
            "mixed": torch.where(torch.rand(n, generator=g) < 0.3, -1, torch.where(torch.rand(n, generator=g) < 0.1, v, skew))}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["uniform", "skewed", "one", "padding", "mixed"])
@pytest.mark.parametrize("n,v,d", [(1, 1, 1), (1, 300, 33), (65, 7, 520), (700, 2, 9), (3001, 1000, 65),
                                   (20011, 517, 130), (5000, 70001, 24), (130, 40, 4104)])
def test_token_gradient(dtype, kind, n, v, d):
    g = gen(n + v + d)
    tok = token_sets(n, v, g)[kind]
    G = normal((n, d), dtype, g)
    want, mag = ref.lookup_grad(torch.arange(n), tok, torch.ones(n, dtype=torch.float64), G.double(), v, 3.0)
    count = torch.bincount(tok[(tok >= 0) & (tok < v)], minlength=v)[:, None]
    got = sp.embed_grad(tok.to(DEV), G.to(DEV), v, 3.0)
    check(got, want, sums_tol(count, mag, want, dtype), f"gradient {kind}")
    assert torch.equal(got, sp.embed_grad(tok.int().to(DEV), G.to(DEV), v, 3.0))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [1, 64, 250])
@pytest.mark.parametrize("values", [True, False])
def test_csr_gradient(dtype, d, values):
    g = gen(d + 5)
    m, n = 411, 1 << 12
    A, rows, cols, vals = csr(g, m, n, 40, values=values, long_row=900)
    G = normal((m, d), dtype, g)
    want, mag = ref.lookup_grad(rows, cols, vals, G.double(), n, 0.5)
    count = torch.bincount(cols, minlength=n)[:, None]
    got = sp.embed_grad(A, G.to(DEV), n, 0.5)
    check(got, want, sums_tol(count, mag, want, dtype), "csr gradient")
    # strided gradients
    wide = torch.zeros((m, d + 3), dtype=dtype)
    wide[:, 1:1 + d] = G
    assert torch.equal(sp.embed_grad(A, wide.to(DEV)[:, 1:1 + d], n, 0.5), got)


def test_lookup_of_nothing():
    W = torch.randn((5, 12), device=DEV)
    none = torch.zeros(0, dtype=torch.int64, device=DEV)
    assert sp.embed(none, W).shape == (0, 12)
    dW = sp.embed_grad(none, torch.zeros((0, 12), device=DEV), 5)
    assert dW.shape == (5, 12) and not dW.any()
    A = sp.DeviceCSR(3, 5, torch.zeros(4, dtype=torch.int64, device=DEV), none.int(), None, 0)
    assert not sp.embed(A, W).any()
    assert not sp.embed_grad(A, torch.ones((3, 12), device=DEV), 5).any()
    assert sp.embed_grad(none, torch.zeros((0, 12), device=DEV), 0).shape == (0, 12)
    assert sp.embed(torch.zeros(3, dtype=torch.int64, device=DEV), W[:, :0]).shape == (3, 0)


def test_lookup_and_gradient_are_adjoint():
    g = gen(3)
    A, rows, cols, vals = csr(g, 200, 90, 20, long_row=700)
    W, G = normal((90, 77), torch.float32, g).to(DEV), normal((200, 77), torch.float32, g).to(DEV)
    left = (sp.embed(A, W, 0.7).double() * G.double())
    right = (W.double() * sp.embed_grad(A, G, 90, 0.7).double())
    # both are the same sum of w W G over entries and columns
    terms = 0.7 * float((W.double()[cols.to(DEV)] * G.double()[rows.to(DEV)]).mul_(vals.to(DEV)[:, None]).abs().sum())
    assert abs(float(left.sum() - right.sum())) <= 800 * U * terms


def test_csr_pointers_out_of_order_stay_inside():
    # not canonical: values are meaningless, accesses are not
    W = torch.randn((50, 40), device=DEV)
    rp = torch.tensor([0, 90, 10, 1 << 40, -5, 100], dtype=torch.int64, device=DEV)
    ci = torch.randint(-5, 60, (100,), dtype=torch.int32, device=DEV)
    A = sp.DeviceCSR(5, 50, rp, ci, None, 100)
    assert sp.embed(A, W).shape == (5, 40)
    assert sp.embed_grad(A, torch.randn((5, 40), device=DEV), 50).shape == (50, 40)
    S = torch.randn((5, 50), device=DEV)
    B = sp.DeviceCSR(5, 50, rp, ci, torch.rand(100, device=DEV), 100)
    loss, grad = sp.distill_grad(S, B)
    assert loss.shape == (5,) and grad.shape == (5, 50)
    torch.cuda.synchronize()


# ---- layer norm

NORM_D = [1, 2, 7, 64, 65, 511, 513, 1001, 2050, 4096, 4099, 8200, 16500, 33000]


def norm_inputs(m, d, dtype, pdtype, seed):
    g = gen(seed)
    x = torch.randn((m, d), generator=g) * (torch.rand((m, 1), generator=g) * 3 + 0.2) + torch.randn((m, 1), generator=g)
    if m > 3:
        x[1] = 2.5            # no variance
        x[2] += 60.0          # a mean far from 0
    return x.to(dtype), normal((d,), pdtype, g), normal((d,), pdtype, g), g


def norm_tols(x, mean, rstd):
    # error of h = (x - mean) rstd: the mean's K u max|x|, the variance's
    # relative K u (and the mean's error squared, below it)
    big = x.abs().amax(1, keepdim=True)
    h = (x - mean[:, None]) * rstd[:, None]
    return h, K * U * (big * rstd[:, None] * (1 + h.abs()) + h.abs())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", NORM_D + [70000])
@pytest.mark.parametrize("params", ["same", "f32", "weight", "none"])
def test_layer_norm(dtype, d, params):
    m = 9
    pdtype = torch.float32 if params == "f32" else dtype
    x, w, b, _ = norm_inputs(m, d, dtype, pdtype, d)
    W = None if params == "none" else w
    B = None if params in ("none", "weight") else b
    wd = torch.ones(d, dtype=torch.float64) if W is None else w.double()
    bd = torch.zeros(d, dtype=torch.float64) if B is None else b.double()
    y0, mean0, rstd0 = ref.layer_norm(x.double(), wd, bd, 1e-5)
    y, mean, rstd = sp.layer_norm(x.to(DEV), None if W is None else W.to(DEV), None if B is None else B.to(DEV))
    h, tol = norm_tols(x.double(), mean0, rstd0)
    check(mean, mean0, K * U * x.double().abs().amax(1), "mean")
    big = x.double().abs().amax(1)
    check(rstd, rstd0, rstd0 * (K * U * 2 + (K * U * big * rstd0) ** 2), "rstd")
    check(y, y0, tol * wd.abs() + 4 * U * bd.abs() + ROUND[dtype] * y0.abs() + TINY[dtype], "y")
    # rows of a wider tensor, three dimensions
    wide = torch.zeros((m, d + 3), dtype=dtype, device=DEV)
    wide[:, 1:1 + d] = x.to(DEV)
    y2 = sp.layer_norm(wide[:, 1:1 + d], None if W is None else W.to(DEV), None if B is None else B.to(DEV))[0]
    y3 = sp.layer_norm(x.to(DEV).view(3, 3, d), None if W is None else W.to(DEV), None if B is None else B.to(DEV))
    assert torch.equal(y2, y) and torch.equal(y3[0].view(m, d), y) and y3[1].shape == (3, 3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", NORM_D)
@pytest.mark.parametrize("m", [1, 5, 1300])
def test_layer_norm_gradient(dtype, d, m):
    if m * d > 6_000_000:
        m = 300
    pdtype = torch.float32 if d % 2 else dtype
    x, w, b, g = norm_inputs(m, d, dtype, pdtype, d + m)
    dy = normal((m, d), dtype, g)
    _, mean, rstd = ref.layer_norm(x.double(), w.double(), b.double(), 1e-5)
    mean, rstd = mean.float(), rstd.float()
    X, DY = x.to(DEV), dy.to(DEV)
    got = sp.layer_norm_grad(DY, X, mean.to(DEV), rstd.to(DEV), w.to(DEV), b.to(DEV))
    want = ref.layer_norm_grad(dy.double(), x.double(), mean.double(), rstd.double(), w.double())
    h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    herr = 4 * U * (h.abs() + (x.double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None])
    a = (dy.double() * w.double()).abs()
    tol = rstd.double()[:, None] * (4 * U * a + K * U * a.mean(1, keepdim=True)
                                   + h.abs() * (K * U * (a * h.abs()).mean(1, keepdim=True) + (a * herr).mean(1, keepdim=True))
                                   + herr * (a * h.abs()).mean(1, keepdim=True))
    check(got[0], want[0], tol + ROUND[dtype] * want[0].abs() + TINY[dtype], "dx")
    ady = dy.double().abs()
    check(got[1], want[1], (m + 8) * U * (ady * h.abs()).sum(0) + (ady * herr).sum(0) + ROUND[pdtype] * want[1].abs() + TINY[pdtype], "dweight")
    check(got[2], want[2], (m + 8) * U * ady.sum(0) + ROUND[pdtype] * want[2].abs() + TINY[pdtype], "dbias")
    again = sp.layer_norm_grad(DY, X, mean.to(DEV), rstd.to(DEV), w.to(DEV), b.to(DEV))
    assert all(torch.equal(p, q) for p, q in zip(got, again))
    # parameters left out; strided rows
    wide = torch.zeros((m, d + 3), dtype=dtype, device=DEV)
    wide[:, 1:1 + d] = X
    part = sp.layer_norm_grad(DY, wide[:, 1:1 + d], mean.to(DEV), rstd.to(DEV), w.to(DEV))
    assert part[2] is None and torch.equal(part[0], got[0]) and torch.equal(part[1], got[1])
    plain = sp.layer_norm_grad(DY, X, mean.to(DEV), rstd.to(DEV))
    assert plain[1] is None and plain[2] is None


def test_layer_norm_of_nothing():
    x = torch.zeros((0, 40), device=DEV)
    w, b = torch.ones(40, device=DEV), torch.ones(40, device=DEV)
    y, mean, rstd = sp.layer_norm(x, w, b)
    assert y.shape == (0, 40) and mean.shape == (0,)
    dx, dw, db = sp.layer_norm_grad(x, x, mean, rstd, w, b)
    assert dx.shape == (0, 40) and not dw.any() and not db.any()


@pytest.mark.parametrize("d", [5, 333])
def test_layer_norm_gradient_against_differences(d):
    x, w, b, g = norm_inputs(4, d, torch.float32, torch.float32, 11)
    x, w, b = x[[0, 3]].double(), w.double(), b.double()
    dy = torch.randn((2, d), generator=g).double()
    _, mean, rstd = sp.layer_norm(x.float().to(DEV))
    dx, dw, db = sp.layer_norm_grad(dy.float().to(DEV), x.float().to(DEV), mean, rstd, w.float().to(DEV), b.float().to(DEV))

    def f(x, w, b):
        return float((ref.layer_norm(x, w, b, 1e-5)[0] * dy.float().double()).sum())

    step = 1e-5
    for arg, grad in ((0, dx), (1, dw), (2, db)):
        base = [x.float().double(), w.float().double(), b.float().double()]
        for j in range(0, base[arg].numel(), max(1, base[arg].numel() // 9)):
            up, down = [t.clone() for t in base], [t.clone() for t in base]
            up[arg].view(-1)[j] += step
            down[arg].view(-1)[j] -= step
            diff = (f(*up) - f(*down)) / (2 * step)
            # central differences: the third derivative's step^2 and the sums' rounding / step
            assert abs(float(grad.view(-1)[j]) - diff) <= 1e-4 * (1 + abs(diff))


# ---- distillation

def distill_inputs(m, v, k, dtype, seed, masked=True):
    g = gen(seed)
    s = torch.randn((m, v), generator=g) * 3
    if masked and v > 4:
        s[:, torch.randperm(v, generator=g)[: v // 8]] = -math.inf
    s = s.to(dtype)
    cols = torch.stack([torch.randperm(v, generator=g)[:k] for _ in range(m)]) if k <= v else torch.randint(0, v, (m, k), generator=g)
    vals = normal((m, k), dtype, g, 2.0)
    if masked:
        # no teacher mass where the student has none
        vals = torch.where(s.gather(1, cols) == -math.inf, torch.full((), -math.inf, dtype=dtype), vals)
    return s, cols, vals, g


def check_distill(s, per_row, T, weight, loss, grad, what, skip=()):
    """per_row: (columns, values) of every row."""
    m, v = s.shape
    dtype = s.dtype
    for r in range(m):
        if r in skip:
            continue
        cols, vals = per_row[r]
        l0, g0, q, p, mag = ref.distill_row(s[r].double(), cols, vals.double(), T)
        tol = T * T * (8 * mag + K) * U
        if l0 == math.inf:
            assert float(loss[r]) == math.inf, (what, r)
        else:
            assert abs(float(loss[r]) - l0) <= tol + 4 * U * abs(l0), (what, r, float(loss[r]), l0, tol)
        if grad is None:
            continue
        w = 1.0 if weight is None else float(weight[r])
        z = torch.where(q > 0, (s[r].double() - s[r].double().max()).abs() / T, 0.0)
        t = vals.double() / T
        t = t[t > t.max() - 800] if t.numel() else t  # (the others have no mass)
        spread = float(t.max() - t.min()) if t.numel() else 0.0
        tol = abs(w) * T * U * (q * (4 * z + K) + p * (4 * spread + K + len(cols)))
        check(grad[r], w * g0, tol + ROUND[dtype] * (w * g0).abs() + abs(w) * T * 2.0 ** -120 + TINY[dtype], f"{what} row {r}")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,v,k", [(1, 1, 1), (2, 5, 5), (3, 8, 1), (5, 1000, 16), (2, 2049, 300), (4, 8193, 64),
                                   (3, 32768, 40), (2, 50021, 20), (1, 131072, 64), (300, 1111, 8), (2, 140001, 33)])
@pytest.mark.parametrize("T", [0.5, 3.0])
def test_distill_pair(dtype, m, v, k, T):
    s, cols, vals, g = distill_inputs(m, v, k, dtype, v + k)
    w = torch.rand(m, generator=g) - 0.3
    if m > 2:
        w[1] = 0.0
    S, teacher = s.to(DEV), (vals.to(DEV), cols.to(DEV))
    loss, grad = sp.distill_grad(S, teacher, T, w.to(DEV))
    rows = [(cols[r], vals[r]) for r in range(m)]
    check_distill(s, rows, T, w, loss.cpu(), grad.cpu(), "pair")
    check_distill(s, rows, T, None, sp.distill(S, teacher, T).cpu(), None, "loss")
    again = sp.distill_grad(S, (teacher[0], teacher[1].int()), T, w.to(DEV))
    assert torch.equal(again[0], loss) and torch.equal(again[1], grad)
    # a slice of wider logits and a teacher with padding
    wide = torch.zeros((m, v + 3), dtype=dtype, device=DEV)
    wide[:, 1:1 + v] = S
    more = torch.cat([cols, torch.full((m, 2), -1), torch.full((m, 1), v)], 1)
    extra = torch.cat([vals, torch.full((m, 3), 30.0, dtype=dtype)], 1)
    padded = sp.distill_grad(wide[:, 1:1 + v], (extra.to(DEV), more.to(DEV)), T, w.to(DEV))
    check_distill(s, rows, T, w, padded[0].cpu(), padded[1].cpu(), "padded")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,v,most", [(40, 300, 20), (13, 8200, 500), (6, 50021, 9000)])
def test_distill_csr(dtype, m, v, most):
    g = gen(v)
    lens = torch.randint(0, min(most, v) + 1, (m,), generator=g)
    lens[0], lens[m - 1] = 0, 1
    cols = [torch.randperm(v, generator=g)[: int(n)].sort().values for n in lens]
    vals = [torch.rand(int(n), generator=g) for n in lens]
    rp = torch.zeros(m + 1, dtype=torch.int64)
    rp[1:] = lens.cumsum(0)
    T = sp.DeviceCSR(m, v, rp.to(DEV), torch.cat(cols).int().to(DEV), torch.cat(vals).to(DEV), int(rp[-1]))
    s = normal((m, v), dtype, g, 2.0)
    loss, grad = sp.distill_grad(s.to(DEV), T, 0.25)
    check_distill(s, list(zip(cols, vals)), 0.25, None, loss.cpu(), grad.cpu(), "csr")
    assert float(loss[0]) == 0.0 and not grad[0].any()
    assert torch.equal(sp.distill(s.to(DEV), T, 0.25), loss)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("v", [37, 9000, 60000])
def test_distill_edges(dtype, v):
    """Rows without mass, lowest values, repeated columns, NaN and infinities."""
    s, cols, vals, g = distill_inputs(10, v, 6, dtype, v, masked=False)
    low = torch.finfo(dtype).min
    inf, nan = math.inf, math.nan
    s[0] = -inf                                # no logits
    vals[1] = -inf                             # no teacher mass
    cols[2] = -1                               # no entries
    s[3, 5:] = low                             # masked by the lowest value
    cols[3, :5] = torch.arange(5)
    vals[3, 5] = -inf
    vals[4, 2:] = low
    cols[5] = cols[5, 0]                       # one column, listed often
    s[6, cols[6, 1]] = -inf                    # teacher mass where the student has none
    s[7, v // 2] = nan
    s[8] = -inf
    s[8, cols[8, 0]] = 1.5                     # all of the student's mass in one column
    vals[8, 1:] = -inf
    s[9, 0] = inf
    w = torch.ones(10)
    loss, grad = sp.distill_grad(s.to(DEV), (vals.to(DEV), cols.to(DEV)), 1.0, w.to(DEV))
    loss, grad = loss.cpu(), grad.cpu()
    check_distill(s, [(cols[r], vals[r]) for r in range(10)], 1.0, w, loss, grad, "edges", skip=(7, 9))
    for r in (7, 9):
        assert math.isnan(float(loss[r])) and grad[r].isnan().any()
    for r in (0, 1, 2):
        assert float(loss[r]) == 0.0 and not grad[r].any()
    assert float(loss[6]) == inf and not grad[6].isnan().any()
    # weight 0: a gradient of zeros whatever the row holds, and only there
    w[[6, 7, 9]] = 0.0
    grad2 = sp.distill_grad(s.to(DEV), (vals.to(DEV), cols.to(DEV)), 1.0, w.to(DEV))[1].cpu()
    assert not grad2[[6, 7, 9]].any()
    keep = [0, 1, 2, 3, 4, 5, 8]
    assert torch.equal(grad2[keep], grad[keep])


def test_distill_of_nothing():
    S = torch.randn((3, 20), device=DEV)
    none = (torch.zeros((3, 0), device=DEV), torch.zeros((3, 0), dtype=torch.int64, device=DEV))
    loss, grad = sp.distill_grad(S, none)
    assert not loss.any() and not grad.any()
    loss, grad = sp.distill_grad(S[:0], (none[0][:0], none[1][:0]))
    assert loss.shape == (0,) and grad.shape == (0, 20)
    wide = (torch.zeros((3, 2), device=DEV), torch.zeros((3, 2), dtype=torch.int64, device=DEV))
    loss, grad = sp.distill_grad(S[:, :0], wide)  # (every entry is padding)
    assert not loss.any() and grad.shape == (3, 0)


def test_distill_gradient_against_differences():
    s, cols, vals, g = distill_inputs(3, 50, 7, torch.float32, 4)
    w = torch.tensor([0.5, 1.0, -2.0])
    grad = sp.distill_grad(s.to(DEV), (vals.to(DEV), cols.to(DEV)), 2.0, w.to(DEV))[1].cpu().double()
    step = 1e-5
    for r in range(3):
        for j in range(0, 50, 7):
            up, down = s[r].double().clone(), s[r].double().clone()
            up[j] += step
            down[j] -= step
            diff = 0.0 if s[r, j] == -math.inf else float(w[r]) * (
                ref.distill_row(up, cols[r], vals[r].double(), 2.0)[0] - ref.distill_row(down, cols[r], vals[r].double(), 2.0)[0]) / (2 * step)
            assert abs(float(grad[r, j]) - diff) <= 1e-5 * (1 + abs(diff))


# ---- sizes, streams, graphs

def test_offsets_past_32_bits():
    v, d = (1 << 20) + 77, 4104
    W = torch.empty((v, d), dtype=torch.bfloat16, device=DEV)
    W[-3:] = torch.randn((3, d), device=DEV).bfloat16()
    tok = torch.tensor([v - 1, v - 3, v], device=DEV)
    got = sp.embed(tok, W, 2.0)
    assert torch.equal(got[:2], (W[[v - 1, v - 3]].float() * 2).bfloat16()) and not got[2].any()
    # the gradient of that table, written whole
    G = torch.randn((3, d), device=DEV).bfloat16()
    del W
    dW = sp.embed_grad(tok, G, v, 1.0)
    assert torch.equal(dW[v - 1], G[0]) and torch.equal(dW[v - 3], G[1])
    assert not dW[v - 2].any() and not dW[:: (v // 49)].any()
    del dW
    # rows of logits past 2^32 elements
    m, v = 33001, 131072
    S = torch.zeros((m, v), dtype=torch.bfloat16, device=DEV)
    S[-1] = torch.randn(v, device=DEV).bfloat16()
    vals = torch.zeros((m, 2), device=DEV)
    cols = torch.tensor([[1, v - 1]], device=DEV).expand(m, 2).contiguous()
    loss, grad = sp.distill_grad(S, (vals, cols))
    last = S[-1:].clone()
    loss1, grad1 = sp.distill_grad(last, (vals[-1:], cols[-1:]))
    # (rows alone may be split over more workgroups: sums in another order)
    assert abs(float(loss[-1] - loss1[0])) <= K * U * 16
    check(grad[-1], ref.f64(grad1[0]), 2 * ROUND[torch.bfloat16] * ref.f64(grad1[0]).abs() + 1e-30, "last row")
    uniform = math.log(v / 2)
    assert abs(float(loss[m // 2]) - uniform) <= K * U * 16 and abs(float(loss[0]) - uniform) <= K * U * 16


def test_side_stream_and_graph():
    g = gen(9)
    v, d, n = 500, 264, 300
    W, G = normal((v, d), torch.bfloat16, g).to(DEV), normal((n, d), torch.bfloat16, g).to(DEV)
    w, b = torch.ones(d, device=DEV), torch.zeros(d, device=DEV)
    tok = torch.randint(-1, v, (n,), generator=g).to(DEV)
    S = normal((n, v), torch.bfloat16, g).to(DEV)
    teacher = tuple(t.to(DEV) for t in torch.topk(torch.randn((n, v), generator=g), 9))

    def step():
        h = sp.embed(tok, W, 4.0)
        y, mean, rstd = sp.layer_norm(h, w, b)
        loss, dS = sp.distill_grad(S, teacher, 2.0)
        dh, dw, db = sp.layer_norm_grad(G, h, mean, rstd, w, b)
        dW = sp.embed_grad(tok, dh, v, 4.0)
        return y, loss, dS, dw, db, dW

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        tok.copy_(torch.randint(-1, v, (n,), generator=g).to(DEV))
        S.copy_(normal((n, v), torch.bfloat16, g).to(DEV))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), k
