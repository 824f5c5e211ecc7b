"""Inputs that require a gradient: the forward calls, which autograd does not
record, refuse them while gradients are recorded.  (No device is touched: the
check comes before that of the device, which is what refuses host tensors.)"""
import pytest
import torch

import paper_2608_09713_amd as sp


def calls():
    x, p = torch.zeros((4, 8)), torch.zeros((4, 8), requires_grad=True)
    tok = torch.zeros(4, dtype=torch.int64)
    w = torch.ones(8, requires_grad=True)
    rp, ci = torch.zeros(5, dtype=torch.int64), torch.zeros(0, dtype=torch.int32)
    bags = sp.DeviceCSR(4, 4, rp, ci, torch.zeros(0, requires_grad=True), 0)
    rows = sp.DeviceCSR(4, 8, rp, ci, torch.zeros(0, requires_grad=True), 0)
    return [(sp.embed, tok, p), (sp.embed, bags, x), (sp.layer_norm, p), (sp.layer_norm, x, w),
            (sp.layer_norm, x, None, w), (sp.distill, p, (x, x.long())), (sp.distill, x, (p, x.long())),
            (sp.distill, x, rows)]


@pytest.mark.parametrize("k", range(8))
def test_forward_calls_refuse_what_autograd_would_lose(k):
    fn, *args = calls()[k]
    with pytest.raises(RuntimeError, match=fn.__name__ + "_grad"):
        fn(*args)
    # nothing is lost where nothing is recorded
    with torch.no_grad(), pytest.raises(TypeError, match="device"):
        fn(*args)


def test_gradient_calls_take_them():
    # (their results are the gradients, to be passed on by the caller)
    p, tok = torch.zeros((4, 8), requires_grad=True), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: sp.embed_grad(tok, p, 16), lambda: sp.layer_norm_grad(p, p, p[:, 0], p[:, 0]),
                 lambda: sp.distill_grad(p, (p, p.long()))):
        with pytest.raises(TypeError, match="device"):
            call()
