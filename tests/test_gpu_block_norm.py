"""The norms around a block on the GPU against a plain 64-bit form.

Tolerances, fixed from the arithmetic: with u = 2^-24 and r the rounding of the
output's type (2^-24, 2^-11, 2^-8),
- a row's sums have at most 16 terms a thread (32 and more where rows are read
  again: d / 1024), 6 steps in a wavefront and 16 over wavefronts: K = 64 + d /
  1024 covers them with the operations that follow, and a norm, a root of a sum
  of squares, has half of that;
- y has 6 u of its second term and u of both; h the error of y, that of the norm
  (at most the norm of y's errors over that of y) and K u of itself;
- the gradient's errors are carried along by the reference in units of u, sums
  over n rows with (n + 8) u of their magnitudes.
"""
import pytest
import torch

import paper_2608_09713_amd as sp
from tests import training_reference as ref
from tests.test_gpu_rows import DEV, DTYPES, ROUND, TINY, U, check, gen, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    sp.library()


def K(d):
    return 64 + d / 1024


def inputs(m, d, dtype, pdtype, g_rows, gdtype, normed, seed=0):
    g = gen(seed + 31 * m + d)
    x, b = normal((m, d), dtype, g, 2.0), normal((m, d), dtype, g, 1.5)
    gate = None if g_rows is None else normal((g_rows, d), gdtype, g, 0.7)
    post = (torch.randn(d, generator=g) * 0.2 + 1).to(pdtype) if normed else None
    pre = (torch.randn(d, generator=g) * 0.2 + 1).to(pdtype)
    return x, b, gate, post, pre, g


def wide(gate, m, d):
    if gate is None:
        return torch.ones((m, d), dtype=torch.float64)
    return gate.double().repeat_interleave(m // gate.shape[0], 0)


def on(t):
    return None if t is None else t.to(DEV)


def run(m, d, dtype, pdtype, g_rows, gdtype, normed, scale=0.75, eps=1e-5, no_dy=False):
    x, b, gate, post, pre, g = inputs(m, d, dtype, pdtype, g_rows, gdtype, normed)
    one = torch.ones(d, dtype=torch.float64)
    full = wide(gate, m, d)
    pd, qd = one if post is None else post.double(), pre.double()
    y, h, r1, r2, term = ref.block_norm(x.double(), b.double(), full, scale, pd, qd, normed, eps)
    args = (on(x), on(b), on(gate), scale, on(post), on(pre), normed, eps)
    got = sp.block_norm(*args)
    k, r = K(d), ROUND[dtype]
    ey = (k / 2 + 6) * U * term.abs() + U * (x.double().abs() + term.abs())
    check(got[0], y, ey + r * (y.abs() + ey) + TINY[dtype], "y")
    en = ey.norm(dim=1, keepdim=True) / (y.norm(dim=1, keepdim=True) + 1e-300) + k * U
    eh = (r2 * qd.abs() * ey) + h.abs() * (en + 4 * U)
    check(got[1], h, eh + r * (h.abs() + eh) + TINY[dtype], "h")
    if normed:
        check(got[2], r1[:, 0], k * U * r1[:, 0], "rstd_post")
    else:
        assert got[2] is None
    check(got[3], r2[:, 0], en[:, 0] * r2[:, 0] + 2 * U * r2[:, 0], "rstd_pre")
    assert all(torch.equal(p, q) for p, q in zip(got, sp.block_norm(*args)) if p is not None)

    dy = None if no_dy else normal((m, d), dtype, g)
    dh = normal((m, d), dtype, g)
    gy, r1f, r2f = got[0].cpu(), None if got[2] is None else got[2].cpu(), got[3].cpu()
    zero = torch.zeros((m, d), dtype=torch.float64)
    want = ref.block_norm_grad(zero if dy is None else dy.double(), dh.double(), gy.double(), b.double(),
                               r1f.double()[:, None] if normed else torch.ones((m, 1), dtype=torch.float64),
                               r2f.double()[:, None], full, scale, pd, qd, normed,
                               1 if g_rows is None else m // g_rows, k)
    gargs = (on(dy), on(dh), on(gy), on(b), on(r1f), on(r2f), on(gate), scale, on(post), on(pre))
    grads = sp.block_norm_grad(*gargs)
    types = dict(dx=dtype, db=dtype, dgate=gdtype, dpost=pdtype, dpre=pdtype)
    for name, got_g in zip(("dx", "db", "dgate", "dpost", "dpre"), grads):
        if got_g is None:
            assert (name == "dgate" and gate is None) or (name == "dpost" and not normed)
            continue
        w, e = want[name]
        rr = ROUND[types[name]]
        e = e * U
        check(got_g.reshape(w.shape), w, e + rr * (w.abs() + e) + TINY[types[name]], name)
    again = sp.block_norm_grad(*gargs)
    assert all(torch.equal(p, q) for p, q in zip(grads, again) if p is not None)


WIDTHS = [1, 3, 7, 8, 9, 31, 64, 130, 250, 512, 520, 1001, 4104, 8192, 8200, 17000]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_widths(dtype, d):
    f32 = torch.float32
    run(37, d, dtype, dtype, 1, dtype, True)
    run(1, d, dtype, f32, 1, f32, False)
    run(36, d, dtype, dtype, 36, dtype, True)
    run(36, d, dtype, f32, 4, dtype, True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,d,g_rows", [(1, 64, None), (300, 64, None), (1030, 72, 1), (1030, 72, 2), (1030, 72, 103),
                                        (1024, 1001, 512), (1030, 1001, 515), (32768, 8, 16384), (32768, 3, 32768),
                                        (700, 520, 700), (66, 17000, 33), (40, 17000, 2), (5, 17000, 5), (9, 8200, None)])
def test_gates(dtype, m, d, g_rows):
    run(m, d, dtype, dtype, g_rows, dtype, True)
    run(m, d, dtype, torch.float32, g_rows, torch.float32, False, no_dy=True)


# (more groups than workgroups, of fewer and of more rows than a workgroup takes side
# by side; groups that several workgroups take, and rows of several kinds of threads)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,d,g_rows", [(8192, 64, 4096), (1800, 128, 600), (1200, 1001, 600), (3000, 1001, 600),
                                        (64, 4096, 16), (1100, 4096, 550), (300, 8192, 150), (140, 9000, 70),
                                        (24, 9000, 3), (520, 8200, 260)])
def test_many_groups(dtype, m, d, g_rows):
    run(m, d, dtype, dtype, g_rows, dtype, True)
    run(m, d, dtype, torch.float32, g_rows, torch.float32, False, no_dy=True)


@pytest.mark.parametrize("dtype", DTYPES[1:])
@pytest.mark.parametrize("pdtype", [0, 1])
@pytest.mark.parametrize("gdtype", [0, 1])
def test_types(dtype, pdtype, gdtype):
    types = (torch.float32, dtype)
    for g_rows in (1, 6, 48):
        run(48, 264, dtype, types[pdtype], g_rows, types[gdtype], True, scale=-1.5)


def test_strides_and_leading_dimensions():
    m, d = 24, 100
    x, b, gate, post, pre, g = inputs(m, d, torch.bfloat16, torch.bfloat16, 6, torch.bfloat16, True)
    want = sp.block_norm(on(x), on(b), on(gate), 0.5, on(post), on(pre))
    wide_x = torch.zeros((m, d + 3), dtype=x.dtype, device=DEV)
    wide_b, wide_g = torch.zeros_like(wide_x), torch.zeros((6, d + 1), dtype=x.dtype, device=DEV)
    wide_x[:, 3:], wide_b[:, 1:1 + d], wide_g[:, 1:] = on(x), on(b), on(gate)
    got = sp.block_norm(wide_x[:, 3:], wide_b[:, 1:1 + d], wide_g[:, 1:], 0.5, on(post), on(pre))
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    shaped = sp.block_norm(on(x).view(2, 3, 4, d), on(b).view(2, 3, 4, d), on(gate).view(2, 3, 1, d), 0.5, on(post), on(pre))
    assert shaped[0].shape == (2, 3, 4, d) and shaped[3].shape == (2, 3, 4)
    assert all(torch.equal(p, q.reshape(p.shape)) for p, q in zip(want, shaped))
    dy, dh = on(normal((m, d), x.dtype, g)), on(normal((m, d), x.dtype, g))
    base = sp.block_norm_grad(dy, dh, want[0], on(b), want[2], want[3], on(gate), 0.5, on(post), on(pre))
    wide_h = torch.zeros_like(wide_x)
    wide_h[:, 2:2 + d] = dh
    got = sp.block_norm_grad(dy, wide_h[:, 2:2 + d], want[0], wide_b[:, 1:1 + d], want[2], want[3], wide_g[:, 1:], 0.5,
                             on(post), on(pre))
    assert all(torch.equal(p, q) for p, q in zip(base, got))
    got = sp.block_norm_grad(dy.view(2, 12, d), dh.view(2, 12, d), want[0].view(2, 12, d), on(b).view(2, 12, d),
                             want[2].view(2, 12), want[3].view(2, 12), on(gate).view(6, 1, d), 0.5, on(post), on(pre))
    assert got[2].shape == (6, 1, d) and all(torch.equal(p, q.reshape(p.shape)) for p, q in zip(base, got))


def test_no_weights_and_no_rows():
    x, b = torch.randn((5, 40), device=DEV), torch.randn((5, 40), device=DEV)
    y, h, r1, r2 = sp.block_norm(x, b)
    ones = torch.ones(40, device=DEV)
    same = sp.block_norm(x, b, ones, 1.0, ones, ones)
    assert torch.equal(y, same[0]) and torch.equal(h, same[1])
    got = sp.block_norm_grad(x, b, y, b, r1, r2)
    assert got[2] is None and got[3] is None and got[4] is None
    full = sp.block_norm_grad(x, b, y, b, r1, r2, ones, 1.0, ones, ones)
    assert torch.equal(got[0], full[0]) and torch.equal(got[1], full[1])
    e, none = torch.empty((0, 40), device=DEV), torch.empty(0, device=DEV)
    y, h, r1, r2 = sp.block_norm(e, e, ones, 1.0, ones, ones)
    assert y.shape == h.shape == (0, 40) and r2.shape == (0,)
    for gate in (ones, None, torch.ones((0, 40), device=DEV)):
        got = sp.block_norm_grad(e, e, e, e, none, none, gate, 1.0, ones, ones)
        assert not got[3].any() and not got[4].any() and (gate is None or not got[2].any())


def test_infinities_stay_in_their_row():
    x, b = torch.randn((6, 200), device=DEV), torch.randn((6, 200), device=DEV)
    clean = sp.block_norm(x, b)
    x[2, 5], b[4, 7] = float("inf"), float("nan")
    got = sp.block_norm(x, b)
    keep = [0, 1, 3, 5]
    assert all(torch.equal(p[keep], q[keep]) for p, q in zip(clean, got))
    assert torch.isnan(got[1][2]).any() and torch.isnan(got[0][4]).all()


def test_gradient_against_differences():
    m, d, per = 12, 40, 3
    x, b, gate, post, pre, g = inputs(m, d, torch.float32, torch.float32, m // per, torch.float32, True)
    a, c = torch.randn((m, d), generator=g), torch.randn((m, d), generator=g)
    y, h, r1, r2 = sp.block_norm(on(x), on(b), on(gate), 0.5, on(post), on(pre), True, 1e-3)
    grads = sp.block_norm_grad(on(a), on(c), y, on(b), r1, r2, on(gate), 0.5, on(post), on(pre))
    start = [t.double() for t in (x, b, gate, post, pre)]
    ways = [torch.randn(t.shape, generator=g).double() for t in start]

    def value(e):
        x, b, gate, post, pre = (t + e * w for t, w in zip(start, ways))
        y, h, *_ = ref.block_norm(x, b, gate.repeat_interleave(per, 0), 0.5, post, pre, True, 1e-3)
        return float((y * a.double()).sum() + (h * c.double()).sum())

    e = 1e-5
    slope = (value(e) - value(-e)) / (2 * e)
    parts = [(t.cpu().double() * w) for t, w in zip(grads, ways)]
    assert abs(float(sum(p.sum() for p in parts)) - slope) <= 1e-5 * float(sum(p.abs().sum() for p in parts))
