"""Forward-mode derivatives of the operators' inputs: calls that would lose them
refuse them, on the host."""
import pytest
import torch
import torch.autograd.forward_ad as fw

import paper_2608_09713_amd as sp

X, W, ROW = torch.zeros((4, 8)), torch.zeros((16, 8)), torch.ones(8)
TOKENS = torch.zeros(4, dtype=torch.int64)


def csr(values):
    return sp.DeviceCSR(4, 8, torch.zeros(5, dtype=torch.int64), torch.zeros(0, dtype=torch.int32), values, 0)


def teacher(values):
    return values, torch.zeros((4, 2), dtype=torch.int64)


CALLS = {
    "embed": (lambda f: sp.embed(TOKENS, f(W)), lambda f: sp.embed(csr(f(ROW)), W)),
    "layer_norm": (lambda f: sp.layer_norm(f(X)), lambda f: sp.layer_norm(X, f(ROW)), lambda f: sp.layer_norm(X, ROW, f(ROW))),
    "distill": (lambda f: sp.distill(f(X), teacher(torch.zeros((4, 2)))), lambda f: sp.distill(X, teacher(f(torch.zeros((4, 2))))),
                lambda f: sp.distill(X, csr(f(ROW)))),
    "linear_cross_entropy": (lambda f: sp.linear_cross_entropy(f(X), W, TOKENS), lambda f: sp.linear_cross_entropy(X, f(W), TOKENS)),
    "block_norm": (lambda f: sp.block_norm(f(X), X), lambda f: sp.block_norm(X, f(X)), lambda f: sp.block_norm(X, X, f(ROW)),
                   lambda f: sp.block_norm(X, X, post=f(ROW)), lambda f: sp.block_norm(X, X, pre=f(ROW))),
}


@pytest.mark.parametrize("name,k", [(n, k) for n, c in CALLS.items() for k in range(len(c))])
def test_tangents_are_refused(name, k):
    call = CALLS[name][k]
    with fw.dual_level():
        for grad in (True, False):
            with torch.set_grad_enabled(grad), pytest.raises(RuntimeError, match="tangent"):
                call(lambda t: fw.make_dual(t, torch.ones_like(t)))
        # (inputs without one are taken up to the next check)
        with pytest.raises(TypeError, match="device"):
            call(lambda t: t)
    with pytest.raises(TypeError, match="device"):
        call(lambda t: t)
