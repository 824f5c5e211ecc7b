"""What a training step's operators refuse, on the host: no device is touched,
neither by the C-ABI's checks nor by the binding's."""
import ctypes

import pytest
import torch

import paper_2608_09713_amd as sp
from tests.test_rows_refusals import INVALID, P, SHAPE, csr, dense, lib, ref, tokens  # noqa: F401


def test_linear_cross_entropy(lib):  # noqa: F811
    x, w, t = dense(4, 8), dense(16, 8), tokens()

    def loss(X=x, W=w, T=t, scale=1.0, out=P, lse=P):
        return lib.spsyrk_linear_cross_entropy(ref(X), ref(W), ref(T), scale, None, None, out, lse)

    def grad(X=x, W=w, T=t, scale=1.0, weight=P, out=P, dX=x, dW=w):
        return lib.spsyrk_linear_cross_entropy_grad(ref(X), ref(W), ref(T), scale, weight, None, None, out, ref(dX),
                                                    ref(dW))

    for bad in (dict(X=None), dict(W=None), dict(T=None), dict(X=dense(4, 9)), dict(W=dense(16, 8, dt=1)),
                dict(X=dense(4, 8, ld=7)), dict(X=dense(4, 8, p=P + 2)), dict(X=dense(4, 8, dt=3)), dict(W=dense(15, 8)),
                dict(T=tokens(m=5)), dict(T=tokens(n=17)), dict(T=tokens(per=2)), dict(T=tokens(values=P)), dict(T=csr()),
                dict(T=tokens(p=None)), dict(T=tokens(p=P + 4)), dict(T=tokens(idx_bytes=2)),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(out=None), dict(out=P + 2),
                dict(X=dense(4, 0), W=dense(16, 0)), dict(W=dense(0, 8), T=tokens(n=0))):
        assert loss(**bad) == INVALID, bad
        assert lib.spsyrk_last_error_detail()
        assert grad(**bad) == INVALID, bad
    assert loss(lse=P + 2) == INVALID
    for bad in (dict(dX=None), dict(dW=None), dict(dX=dense(4, 9)), dict(dX=dense(3, 8)), dict(dW=dense(15, 8)),
                dict(dW=dense(16, 8, dt=2)), dict(weight=P + 2)):
        assert grad(**bad) == INVALID, bad
    assert loss(X=dense(1 << 31, 8), T=tokens(m=1 << 31)) == SHAPE


def test_binding():
    x, w, t = torch.zeros((4, 8)), torch.zeros((16, 8)), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(TypeError, match="device"):
        sp.linear_cross_entropy(x, w, t)
    with pytest.raises(TypeError, match="device"):
        sp.linear_cross_entropy_grad(x, w, t)
    with pytest.raises(TypeError):
        sp.linear_cross_entropy(x.double(), w, t)


@pytest.mark.parametrize("k", range(2))
def test_forward_calls_refuse_what_autograd_would_lose(k):
    x, w = torch.zeros((4, 8), requires_grad=k == 0), torch.zeros((16, 8), requires_grad=k == 1)
    t = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(RuntimeError, match="linear_cross_entropy_grad"):
        sp.linear_cross_entropy(x, w, t)
    with torch.no_grad(), pytest.raises(TypeError, match="device"):
        sp.linear_cross_entropy(x, w, t)
    with pytest.raises(TypeError, match="device"):
        sp.linear_cross_entropy_grad(x, w, t)


def test_block_norm(lib):  # noqa: F811
    x = dense(4, 8)

    def fwd(X=x, B=x, gate=None, scale=1.0, post=P, pre=P, pt=0, no_norm=0, eps=1e-6, Y=x, H=x, r1=P, r2=P):
        return lib.spsyrk_block_norm(ref(X), ref(B), ref(gate), scale, post, pre, pt, no_norm, eps, None, ref(Y), ref(H),
                                     r1, r2)

    def bwd(dY=x, dH=x, Y=x, B=x, r1=P, r2=P, gate=None, post=P, pre=P, pt=0, dX=x, dB=x, dgate=None, dpost=P, dpre=P):
        return lib.spsyrk_block_norm_grad(ref(dY), ref(dH), ref(Y), ref(B), r1, r2, ref(gate), 1.0, post, pre, pt, None,
                                          None, ref(dX), ref(dB), ref(dgate), dpost, dpre)

    for bad in (dict(X=None), dict(B=None), dict(Y=None), dict(H=None), dict(B=dense(4, 9)), dict(B=dense(3, 8)),
                dict(Y=dense(4, 8, dt=1)), dict(H=dense(5, 8)), dict(X=dense(4, 8, ld=7)),
                dict(X=dense(4, 0), B=dense(4, 0), Y=dense(4, 0), H=dense(4, 0)), dict(eps=-1.0), dict(eps=float("nan")),
                dict(no_norm=1), dict(r1=None), dict(r2=None), dict(r1=P + 2), dict(r2=P + 1), dict(pt=1), dict(pt=9),
                dict(post=P + 2), dict(pre=P + 3), dict(gate=dense(3, 8)), dict(gate=dense(8, 8)), dict(gate=dense(0, 8)),
                dict(gate=dense(2, 7)), dict(gate=dense(2, 8, dt=1)), dict(gate=dense(2, 8, p=None))):
        assert fwd(**bad) == INVALID, bad
        assert lib.spsyrk_last_error_detail()
    g = dense(2, 8)
    for bad in (dict(dH=None), dict(Y=None), dict(B=None), dict(dX=None), dict(dB=None), dict(dY=dense(4, 9)),
                dict(dH=dense(4, 8, dt=2)), dict(dX=dense(5, 8)), dict(dB=dense(4, 9)), dict(r1=None), dict(r2=None),
                dict(r1=P + 2), dict(r2=P + 2), dict(pt=2), dict(post=P + 1), dict(dpost=P + 2), dict(dpre=P + 1),
                dict(gate=g), dict(dgate=g), dict(gate=g, dgate=dense(4, 8)), dict(gate=dense(3, 8), dgate=dense(3, 8)),
                dict(gate=g, dgate=dense(2, 8, dt=2))):
        assert bwd(**bad) == INVALID, bad


def adam(n=10, **kw):
    t = sp._AdamTensor(n, P, P, None, P, P, P, P)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def test_adamw(lib):  # noqa: F811
    def step(*tensors, pt=0, gt=0, bits=32, count=None, how=True, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, decay=0.1, k=1, scale=None):
        table = (sp._AdamTensor * max(len(tensors), 1))(*tensors)
        s = sp._AdamStep(pt, gt, bits, k, lr, b1, b2, eps, decay, scale)
        return lib.spsyrk_adamw(table if tensors else None, len(tensors) if count is None else count,
                                ctypes.byref(s) if how else None, None)

    assert step() == 0 and step(adam(n=0, param=None)) == 0  # (nothing to do)
    for bad in (dict(how=False), dict(pt=3), dict(pt=0, gt=1), dict(pt=1, gt=2), dict(bits=16), dict(k=0), dict(lr=float("nan")),
                dict(lr=float("inf")), dict(decay=float("nan")), dict(eps=-1e-8), dict(eps=float("inf")), dict(b1=1.0),
                dict(b1=-0.1), dict(b2=1.0), dict(b2=float("nan")), dict(count=-1), dict(scale=P + 2)):
        assert step(adam(), **bad) == INVALID, bad
        assert lib.spsyrk_last_error_detail()
    assert step(count=2) == INVALID
    for bad in (dict(n=-1), dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(param=P + 2),
                dict(grad=P + 1), dict(m=P + 2), dict(v=P + 2)):
        assert step(adam(**bad)) == INVALID, bad
    assert step(adam(n=1 << 33)) == SHAPE
    for bad in (dict(m_scale=None), dict(v_scale=None), dict(m_scale=P + 2), dict(v_scale=P + 1)):
        assert step(adam(**bad), bits=8) == INVALID, bad
    assert step(adam(master=P)) == INVALID                        # (32-bit parameters)
    assert step(adam(master=P), adam(), pt=2, gt=2) == INVALID    # (some with copies)
    assert step(adam(master=P + 2), pt=2, gt=2) == INVALID

    def values(t, m=P, v=P, count=1):
        table, ms, vs = (sp._AdamTensor * 1)(t), (ctypes.c_void_p * 1)(m), (ctypes.c_void_p * 1)(v)
        return lib.spsyrk_adam_values(table, count, ms, vs, None)

    assert values(adam(n=0)) == 0
    for call in (values(adam(), m=None), values(adam(), v=None), values(adam(), m=P + 2), values(adam(m=None)),
                 values(adam(n=-1)), values(adam(m_scale=None)), values(adam(), count=-1),
                 lib.spsyrk_adam_values(None, 1, None, None, None)):
        assert call == INVALID


def test_binding_of_the_others():
    x = torch.zeros((4, 8))
    with pytest.raises(TypeError, match="device"):
        sp.block_norm(x, x)
    with pytest.raises(TypeError, match="device"):
        sp.block_norm_grad(x, x, x, x, x[:, 0], x[:, 0])
    for k in range(4):
        args = [x, x, torch.ones(8), 1.0, torch.ones(8), torch.ones(8)]
        args[(0, 1, 2, 4)[k]] = args[(0, 1, 2, 4)[k]].clone().requires_grad_()
        with pytest.raises(RuntimeError, match="block_norm_grad"):
            sp.block_norm(*args)
    s = sp.adam_state(x)
    with pytest.raises(TypeError, match="device"):
        sp.adamw([x], [x], [s], 1e-3, 1)
    with pytest.raises(ValueError, match="length"):
        sp.adamw([x], [x, x], [s], 1e-3, 1)
    with pytest.raises(ValueError):
        sp.adam_state(x, 16)
    with pytest.raises(TypeError, match="device"):
        sp.adam_values([sp.adam_state(x, 8)])
    assert sp.adam_values([s])[0][0] is s.m
    assert sp.adam_state(torch.zeros(257), 8).m_scale.numel() == 2
    with pytest.raises(TypeError):
        sp.adam_values([sp.AdamState(s.m, s.v.double())])


def test_sizes_past_the_limits(lib):  # noqa: F811
    # (columns of X, rows of W; fewer of those for the gradient, whose exponentials are rows of them)
    def calls(v, d):
        x, w, t = dense(4, d), dense(v, d), tokens(n=v)
        return (lib.spsyrk_linear_cross_entropy(ref(x), ref(w), ref(t), 1.0, None, None, P, P),
                lib.spsyrk_linear_cross_entropy_grad(ref(x), ref(w), ref(t), 1.0, None, None, None, P, ref(x), ref(w)))

    assert calls(16, 1 << 22) == (SHAPE, SHAPE)
    assert calls(1 << 28, 1) == (SHAPE, SHAPE)
    assert calls(1 << 22, 1)[1] == SHAPE
    big = (sp._AdamTensor * 1)()
    big[0].n, big[0].param, big[0].grad, big[0].m, big[0].v = 1 << 33, P, P, P, P
    how = sp._AdamStep(0, 0, 32, 1, 1e-3, 0.9, 0.999, 1e-8, 0.0)
    assert lib.spsyrk_adamw(big, 1, ref(how), None) == SHAPE
