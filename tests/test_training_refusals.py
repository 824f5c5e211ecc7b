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
