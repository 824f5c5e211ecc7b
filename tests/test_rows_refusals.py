"""What the operators between sparse rows and dense rows refuse, on the host:
no device is touched, neither by the C-ABI's checks nor by the binding's."""
import ctypes

import pytest
import torch

import paper_2608_09713_amd as sp

INVALID, SHAPE = 1, 3
P = 1 << 20  # (an address that is never read)


@pytest.fixture(scope="module")
def lib():
    return sp.library()


def dense(m=4, n=8, ld=None, dt=0, p=P):
    return sp._Dense(m, n, n if ld is None else ld, dt, p)


def tokens(m=4, n=16, p=P, per=1, **kw):
    e = sp._Entries(m, n, 0, None, per, per, per, p, 8, 0, None)
    for k, v in kw.items():
        setattr(e, k, v)
    return e


def csr(m=4, n=16, nnz=10, values=None, **kw):
    e = sp._Entries(m, n, nnz, P, 0, 0, 0, P, 4, 0, values)
    for k, v in kw.items():
        setattr(e, k, v)
    return e


def ref(x):
    return None if x is None else ctypes.byref(x)


def embed(lib, A, W, Y):
    return lib.spsyrk_embed(ref(A), ref(W), 1.0, None, None, ref(Y))


def embed_grad(lib, A, G, dW):
    return lib.spsyrk_embed_grad(ref(A), ref(G), 1.0, None, None, ref(dW))


@pytest.mark.parametrize("call", [embed, embed_grad])
def test_lookup(lib, call):
    def dims(A, table, rows):
        return (A, table, rows) if call is embed else (A, rows, table)

    table, rows = dense(16, 8), dense(4, 8)
    for bad in (None, tokens(m=-1), tokens(per=-1), tokens(per=2), tokens(values=P), tokens(idx_bytes=2),
                tokens(idx_stride=-1), tokens(p=None), tokens(p=P + 4), csr(nnz=-1), csr(col_idx=None),
                csr(row_ptr=P + 1), csr(values=P, val_dtype=3), csr(values=P + 2), csr(n=15), tokens(m=5)):
        assert call(lib, *dims(bad, table, rows)) == INVALID, bad
        assert lib.spsyrk_last_error_detail()
    for bad in (tokens(m=1 << 31), tokens(n=1 << 31), csr(nnz=1 << 31)):
        assert call(lib, *dims(bad, table, rows)) == SHAPE
    for bad in (None, dense(16, 8, ld=7), dense(16, 8, dt=3), dense(16, 8, dt=-1), dense(16, 8, p=None),
                dense(16, 8, p=P + 1), dense(16, 8, dt=1), dense(16, 9), dense(15, 8), dense(-1, 8)):
        assert call(lib, *dims(tokens(), bad, rows)) == INVALID, bad
    assert call(lib, *dims(tokens(), dense(16, 1 << 31), dense(4, 1 << 31))) == SHAPE


def norm(lib, X, Y, gamma=P, beta=P, pt=0, eps=1e-5, mean=P, rstd=P):
    return lib.spsyrk_layer_norm(ref(X), gamma, beta, pt, eps, None, ref(Y), mean, rstd)


def norm_grad(lib, G, X, dX, mean=P, rstd=P, gamma=P, pt=0, dgamma=P, dbeta=P):
    return lib.spsyrk_layer_norm_grad(ref(G), ref(X), mean, rstd, gamma, pt, None, None, ref(dX), dgamma, dbeta)


def test_layer_norm(lib):
    x = dense()
    for X, Y in ((None, x), (x, None), (x, dense(n=9)), (x, dense(m=5)), (x, dense(dt=1)), (dense(n=0), dense(n=0))):
        assert norm(lib, X, Y) == INVALID
    for kw in (dict(pt=1), dict(pt=7), dict(eps=-1.0), dict(eps=float("nan")), dict(mean=None), dict(rstd=None),
               dict(gamma=P + 2), dict(beta=P + 1), dict(mean=P + 2)):
        assert norm(lib, x, x, **kw) == INVALID, kw
    for G, X, D in ((None, x, x), (x, None, x), (x, x, None), (dense(n=9), x, x), (x, x, dense(m=3)),
                    (dense(dt=2), x, x)):
        assert norm_grad(lib, G, X, D) == INVALID
    for kw in (dict(pt=2), dict(mean=None), dict(rstd=None), dict(gamma=P + 2), dict(dgamma=P + 2),
               dict(dbeta=P + 3)):
        assert norm_grad(lib, x, x, x, **kw) == INVALID, kw


def test_distill(lib):
    def loss(S, t, T=1.0, out=P):
        return lib.spsyrk_distill(ref(S), ref(t), T, None, None, out)

    def grad(S, t, dS, T=1.0, w=None, out=P):
        return lib.spsyrk_distill_grad(ref(S), ref(t), T, w, None, None, out, ref(dS))

    s, t = dense(4, 16), csr(values=P)
    for S, teacher in ((None, t), (s, None), (s, csr()), (s, csr(m=5, values=P)), (s, csr(n=17, values=P)),
                       (s, tokens(per=3))):
        assert loss(S, teacher) == INVALID
        assert grad(S, teacher, s) == INVALID
    for T in (0.0, -1.0, float("inf"), float("nan")):
        assert loss(s, t, T) == INVALID and grad(s, t, s, T) == INVALID
    assert loss(s, t, out=None) == INVALID and loss(s, t, out=P + 2) == INVALID
    for dS in (None, dense(4, 15), dense(4, 16, dt=1), dense(3, 16)):
        assert grad(s, t, dS) == INVALID
    assert grad(s, t, s, w=P + 1) == INVALID
    assert loss(dense(1 << 30, 16), tokens(m=1 << 30, per=4, values=P)) == SHAPE


def test_distill_temperatures_without_a_reciprocal(lib):
    s, t = dense(4, 16), csr(values=P)
    for T in (1e-40, 1.17e-38, -1e-40):
        assert lib.spsyrk_distill(ref(s), ref(t), T, None, None, P) == INVALID
        assert lib.spsyrk_distill_grad(ref(s), ref(t), T, None, None, None, P, ref(s)) == INVALID


def test_binding():
    x = torch.zeros((4, 8))
    tok = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(TypeError):
        sp.embed(tok, x)                       # host tensors
    with pytest.raises(TypeError):
        sp.embed_grad(tok, x, 16)
    with pytest.raises(TypeError):
        sp.layer_norm(x)
    with pytest.raises(TypeError):
        sp.layer_norm_grad(x, x, x[:, 0], x[:, 0])
    with pytest.raises(TypeError):
        sp.distill(x, (x, x.long()))
    with pytest.raises(TypeError):
        sp.distill_grad(x.double(), (x, x.long()))  # no such element type
    with pytest.raises(AttributeError):
        sp.no_such_call
