"""Lookup, layer norm and distillation on the GPU: the paths that only large
sizes or unusual values take, and the calls together.

Tolerances as in test_gpu_rows.py.
"""
import math

import pytest
import torch

import paper_2608_09713_amd as sp
from tests import rows_reference as ref
from tests.test_gpu_rows import DEV, DTYPES, K, ROUND, TINY, U, check, check_distill, csr, gen, normal, sums_tol

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    sp.library()


# ---- the sort of the table's gradient

@pytest.mark.parametrize("v", [524288, 524289, 3_000_001])
@pytest.mark.parametrize("kind", ["uniform", "one", "mixed"])
def test_token_gradient_over_many_columns(v, kind):
    # up to 2^19 columns two launches sort the tokens, past that passes over digits
    g = gen(v)
    n, d = 5003, 12
    tok = {"uniform": torch.randint(0, v, (n,), generator=g), "one": torch.full((n,), v - 1),
           "mixed": torch.where(torch.rand(n, generator=g) < 0.3, -1,
                                torch.where(torch.rand(n, generator=g) < 0.5, v - 1 - torch.randint(0, 9, (n,), generator=g), v))}[kind]
    G = normal((n, d), torch.float32, g)
    want, mag = ref.lookup_grad(torch.arange(n), tok, torch.ones(n, dtype=torch.float64), G.double(), v, 1.0)
    count = torch.bincount(tok[(tok >= 0) & (tok < v)], minlength=v)[:, None]
    check(sp.embed_grad(tok.to(DEV), G.to(DEV), v), want, sums_tol(count, mag, want, torch.float32), kind)


@pytest.mark.parametrize("n", [63, 1023, 1024, 1025])
@pytest.mark.parametrize("v", [1, 255, 257, 3001, 262_145, 524_288])
def test_token_gradient_of_few_tokens(n, v):
    # up to 1024 tokens one launch sorts them
    g = gen(n + v)
    for tok in (torch.randint(-2, v + 2, (n,), generator=g), torch.full((n,), v - 1), torch.full((n,), v)):
        G = normal((n, 6), torch.float32, g)
        want, mag = ref.lookup_grad(torch.arange(n), tok, torch.ones(n, dtype=torch.float64), G.double(), v, 1.0)
        count = torch.bincount(tok[(tok >= 0) & (tok < v)], minlength=v)[:, None]
        for t in (tok.to(DEV), tok.int().to(DEV)):
            check(sp.embed_grad(t, G.to(DEV), v), want, sums_tol(count, mag, want, torch.float32), "few tokens")


@pytest.mark.parametrize("n", [131072, 131073, 400_009])
def test_token_gradient_of_many_tokens(n):
    # tiles of 1024 tokens up to 2^17 of them, of 4096 past that
    g = gen(n)
    v, d = 3001, 8
    tok = (v * torch.rand(n, generator=g) ** 3).long() - 1
    G = normal((n, d), torch.float32, g)
    want, mag = ref.lookup_grad(torch.arange(n), tok, torch.ones(n, dtype=torch.float64), G.double(), v, 1.0)
    count = torch.bincount(tok[tok >= 0], minlength=v)[:, None]
    got = sp.embed_grad(tok.to(DEV), G.to(DEV), v)
    check(got, want, sums_tol(count, mag, want, torch.float32), "many tokens")
    assert torch.equal(got, sp.embed_grad(tok.int().to(DEV), G.to(DEV), v))


@pytest.mark.parametrize("m,n,most", [(40_000, 9_000, 24), (200_001, 700_000, 20), (260_000, 60_000, 40)])
@pytest.mark.parametrize("values", [True, False])
def test_csr_gradient_of_many_entries(m, n, most, values):
    # the two-launch sort with 4096 entries a tile; more columns, and more
    # entries (over 2^22), than it takes
    g = gen(m)
    A, rows, cols, vals = csr(g, m, n, most, values=values)
    G = normal((m, 4), torch.float32, g)
    want, mag = ref.lookup_grad(rows, cols, vals, G.double(), n, 1.0)
    count = torch.bincount(cols, minlength=n)[:, None]
    check(sp.embed_grad(A, G.to(DEV), n), want, sums_tol(count, mag, want, torch.float32), "many entries")
    W = normal((n, 4), torch.float32, g)
    want, mag = ref.lookup(rows, cols, vals, W.double(), m, 1.0)
    count = torch.bincount(rows, minlength=m)[:, None]
    check(sp.embed(A, W.to(DEV)), want, sums_tol(count, mag, want, torch.float32), "lookup of many entries")


def test_csr_rows_mostly_empty():
    # a tile of entries whose rows' pointers do not fit LDS
    g = gen(8)
    m, n, nnz = 500_000, 300, 20_000
    rows = torch.randint(0, m, (nnz,), generator=g).sort().values
    cols = torch.randint(0, n, (nnz,), generator=g)
    rp = torch.zeros(m + 1, dtype=torch.int64)
    rp[1:] = torch.bincount(rows, minlength=m).cumsum(0)
    A = sp.DeviceCSR(m, n, rp.to(DEV), cols.int().to(DEV), None, nnz)
    G = normal((m, 20), torch.float32, g)
    one = torch.ones(nnz, dtype=torch.float64)
    want, mag = ref.lookup_grad(rows, cols, one, G.double(), n, 1.0)
    count = torch.bincount(cols, minlength=n)[:, None]
    check(sp.embed_grad(A, G.to(DEV), n), want, sums_tol(count, mag, want, torch.float32), "empty rows")


@pytest.mark.parametrize("d", [2, 9, 30, 70, 700])
def test_nan_beside_and_under_padding(d):
    # what padding would have read or been weighted with is NaN or infinite;
    # an infinite weight reaches its own target only
    g = gen(d)
    nan, inf = math.nan, math.inf
    tok = torch.tensor([3, -1, 5, 9, 3, 4, -7], device=DEV)
    W = normal((9, d), torch.float32, g).to(DEV)
    W[[0, 1]] = nan
    y = sp.embed(tok, W, 2.0)
    assert not y[[1, 3, 6]].any() and torch.equal(y[[0, 2, 4, 5]], W[[3, 5, 3, 4]] * 2)
    G = normal((7, d), torch.float32, g).to(DEV)
    G[[1, 3, 6]] = nan
    dW = sp.embed_grad(tok, G, 9)
    assert torch.equal(dW[3], G[0] + G[4]) and torch.equal(dW[4], G[5]) and not dW[[0, 1, 2, 6, 7, 8]].any()
    # CSR: rows of one to nine entries, the padded ones weighted NaN and infinity
    rp = torch.tensor([0, 1, 3, 8, 17, 18], dtype=torch.int64, device=DEV)
    ci = torch.tensor([2, -1, 3, 4, 99, 5, 6, -2, 2, 3, 4, 5, 6, 7, 8, -1, 2, 4], dtype=torch.int32, device=DEV)
    w = torch.tensor([1.0, nan, 1, 1, inf, 1, 1, -inf, 1, 1, 1, 1, 1, 1, 1, nan, 1, inf], device=DEV)
    A = sp.DeviceCSR(5, 9, rp, ci, w, 18)
    y = sp.embed(A, W)
    for r in range(4):
        c = [int(x) for x in ci[int(rp[r]):int(rp[r + 1])] if 0 <= x < 9]
        want = W[c].double().sum(0)
        assert ((y[r].double() - want).abs() <= 12 * U * W[c].double().abs().sum(0)).all()
    assert torch.equal(y[4], W[4] * inf)
    dW = sp.embed_grad(A, torch.ones((5, d), device=DEV), 9)
    assert torch.equal(dW[:, 0].cpu(), torch.tensor([0.0, 0, 3, 2, inf, 2, 2, 1, 1]))


# ---- layer norm over row shapes

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [3, 4, 15, 16, 31, 33, 127, 129, 255, 257, 1023, 1025, 1032, 3080, 5121, 6145, 8193, 12289, 16384, 16385, 32768, 32769])
def test_layer_norm_row_shapes(dtype, d):
    g = gen(d)
    m = 37
    x, dy = normal((m, d), dtype, g, 2.0), normal((m, d), dtype, g)
    w, b = normal((d,), torch.float32, g), normal((d,), torch.float32, g)
    X, DY, W, B = x.to(DEV), dy.to(DEV), w.to(DEV), b.to(DEV)
    y0, mean0, rstd0 = ref.layer_norm(x.double(), w.double(), b.double(), 1e-5)
    y, mean, rstd = sp.layer_norm(X, W, B)
    big = x.double().abs().amax(1, keepdim=True)
    k = 128 * U
    h = (x.double() - mean0[:, None]) * rstd0[:, None]
    check(y, y0, k * (big * rstd0[:, None] * (1 + h.abs()) + h.abs()) * w.double().abs() + 4 * U * b.double().abs()
          + ROUND[dtype] * y0.abs() + TINY[dtype], "y")
    mean, rstd = mean0.float(), rstd0.float()
    got = sp.layer_norm_grad(DY, X, mean.to(DEV), rstd.to(DEV), W, B)
    want = ref.layer_norm_grad(dy.double(), x.double(), mean.double(), rstd.double(), w.double())
    r = rstd.double()[:, None]
    h = (x.double() - mean.double()[:, None]) * r
    herr = 4 * U * (h.abs() + (x.double().abs() + mean.double().abs()[:, None]) * r)
    a = (dy.double() * w.double()).abs()
    ah = (a * h.abs()).mean(1, keepdim=True)
    tol = r * (4 * U * a + k * a.mean(1, keepdim=True) + h.abs() * (k * ah + (a * herr).mean(1, keepdim=True)) + herr * ah)
    check(got[0], want[0], tol + ROUND[dtype] * want[0].abs() + TINY[dtype], "dx")
    ady = dy.double().abs()
    check(got[1], want[1], (m + 8) * U * (ady * h.abs()).sum(0) + (ady * herr).sum(0) + U * want[1].abs(), "dweight")
    check(got[2], want[2], (m + 8) * U * ady.sum(0) + U * want[2].abs(), "dbias")


# ---- distillation

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("v", [60, 5000, 140_001])
@pytest.mark.parametrize("T", [0.25, 1.0, 8.0])
def test_distill_at_the_ends_of_the_type(dtype, v, T):
    """Logits whose quotient by T leaves the floats' range."""
    g = gen(v)
    info = torch.finfo(dtype)
    s = normal((5, v), dtype, g, 2.0)
    s[0] = info.min                                     # all masked by the lowest value: uniform
    s[1] = info.min
    s[1, 7] = info.min / 2                              # one column far above the others
    s[2, 3:9] = info.max                                # several at the largest value
    s[3] = s[3] * 100 if dtype != torch.float16 else s[3] * 50
    cols = torch.stack([torch.randperm(v, generator=g)[:4] for _ in range(5)])
    cols[1, 0], cols[2, 0] = 7, 5
    vals = normal((5, 4), torch.float32, g)
    vals[1, 1:] = -math.inf                             # (no mass where the student has none)
    cols[2, 1:] = torch.tensor([3, 4, 6])
    cols[3, 1:], vals[3, 0] = s[3].float().topk(3).indices, -math.inf
    w = torch.tensor([1.0, 0.5, -1.0, 2.0, 1.0])
    loss, grad = sp.distill_grad(s.to(DEV), (vals.to(DEV), cols.to(DEV)), T, w.to(DEV))
    rows = [(cols[r], vals[r]) for r in range(5)]
    check_distill(s, rows, T, w, loss.cpu(), grad.cpu(), "ends")
    check_distill(s, rows, T, None, sp.distill(s.to(DEV), (vals.to(DEV), cols.to(DEV)), T).cpu(), None, "ends")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("v", [9, 63, 500, 2047, 4100, 8191, 16390, 30001, 65535, 131065])
def test_distill_row_shapes(dtype, v):
    """Rows at every distance from a 16-byte boundary, several rows per workgroup."""
    g = gen(v)
    m = 600 if v < 10_000 else 9
    k = min(v, 30)
    s = normal((m, v), dtype, g, 2.0)
    cols = torch.rand((m, v if v < 10_000 else k), generator=g)
    cols = cols.topk(k).indices if v < 10_000 else (cols * v).long() // k * k + torch.arange(k)
    cols = cols.clamp(max=v - 1)
    vals = normal((m, k), dtype, g)
    w = torch.rand(m, generator=g)
    loss, grad = sp.distill_grad(s.to(DEV), (vals.to(DEV), cols.to(DEV)), 1.0, w.to(DEV))
    assert torch.equal(loss, sp.distill(s.to(DEV), (vals.to(DEV), cols.to(DEV)), 1.0))
    pick = list(range(0, m, max(1, m // 40)))
    check_distill(s[pick], [(cols[r], vals[r]) for r in pick], 1.0, w[pick], loss.cpu()[pick], grad.cpu()[pick], "shapes")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,packs", [(13_001, 26), (13_001, 300), (2600, 2047), (600, 8001), (600, 9251), (600, 11251),
                                     (600, 13251), (300, 16001)])
def test_distill_workgroups_take_many_rows(dtype, m, packs):
    """More rows than the chip holds at once, at every number of packs per thread,
    and rows that lie at other distances from a boundary than the ones before."""
    v = packs * (16 // (torch.finfo(dtype).bits // 8)) - 3
    g = torch.Generator(DEV).manual_seed(packs)
    k = 20
    s = torch.randn((m, v), generator=g, device=DEV).mul_(2.0).to(dtype)
    # (at most one entry a stretch of columns, some of them at the row's ends)
    cols = torch.arange(k, device=DEV) * (v // k) + torch.randint(0, v // k, (m, k), generator=g, device=DEV)
    cols[::2, 0], cols[::2, k - 1] = 0, v - 1
    vals = torch.randn((m, k), generator=g, device=DEV).to(dtype)
    w = torch.rand(m, generator=g, device=DEV)
    w[::7] = 0.0
    loss, grad = sp.distill_grad(s, (vals, cols), 2.0, w)
    assert torch.equal(loss, sp.distill(s, (vals, cols), 2.0))
    pick = sorted({0, 1, 255, 256, 257, m // 2, m // 2 + 1, m - 258, m - 257, m - 2, m - 1} & set(range(m)))
    rows = [(cols[r].cpu(), vals[r].cpu()) for r in pick]
    check_distill(s[pick].cpu(), rows, 2.0, w[pick].cpu(), loss[pick].cpu(), grad[pick].cpu(), "many rows")
    # every row of the gradient sums to nothing, up to the sum of its elements'
    # bars (as in check_distill: z <= 11, a spread of 5 and sums of q and p of 1)
    total, size = torch.empty(m, device=DEV), torch.empty(m, device=DEV)
    for r in range(0, m, 100):
        part = grad[r:r + 100].double()
        total[r:r + 100], size[r:r + 100] = part.sum(1).abs(), part.abs().sum(1)
    bar = ROUND[dtype] * size + w * 2.0 * U * (4 * 11 + K + 4 * 5 + K + k) + v * TINY[dtype]
    assert bool((total <= bar).all()), int((total > bar).sum())


def test_distill_more_entries_than_threads_by_row():
    """Rows of few and of very many entries in one call, in rows held in registers and in longer ones."""
    g = gen(2)
    for v in (700, 20_000, 150_001):
        lens = [3, v // 2, 0, 64, 65, v, 1, 400]
        cols = [torch.randperm(v, generator=g)[:n].sort().values for n in lens]
        vals = [torch.randn(n, generator=g) for n in lens]
        rp = torch.tensor([0] + lens).cumsum(0)
        T = sp.DeviceCSR(len(lens), v, rp.to(DEV), torch.cat(cols).int().to(DEV), torch.cat(vals).to(DEV), int(rp[-1]))
        s = normal((len(lens), v), torch.float32, g, 2.0)
        loss, grad = sp.distill_grad(s.to(DEV), T, 1.5)
        check_distill(s, list(zip(cols, vals)), 1.5, None, loss.cpu(), grad.cpu(), f"rows of {v}")


# ---- together

def test_one_training_step_lowers_the_loss():
    """Rows of overlaps: their bags looked up, normalised, multiplied with the
    reads' own vectors, distilled from the Jaccard rows, and back."""
    import examples.overlap_embedding as example
    losses = example.train(rows=2048, columns=1 << 14, dim=64, steps=6, device=DEV, log=None)
    assert all(math.isfinite(x) for x in losses)
    assert losses[-1] < 0.9 * losses[0]
