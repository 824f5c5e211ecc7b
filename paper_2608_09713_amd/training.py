"""Operators of a training step: the cross entropy of a linear layer over many
columns, forward and backward (C-ABI in ``include/spsyrk.h``).

What ``rows.py`` says of tensors, streams and autograd holds here too: dense
arguments are float32, float16 or bfloat16 rows of one GPU, work is enqueued on
the current stream, gradients are calls of their own, and a forward call refuses
an input whose gradient would be lost.
"""
from __future__ import annotations

import torch

import paper_2608_09713_amd as _sp

from .rows import (_arena, _byref, _check, _like, _on_device, _raw_stream, _rows, _same_device, _tokens, _unrecorded,
                   _vector)


def _linear(x, weight, targets):
    """Arguments of the linear layer's loss: (_Dense of x, of weight, _Entries of targets)."""
    a, w = _rows(x, "x"), _rows(weight, "weight")
    if weight.dim() != 2:
        raise ValueError("weight must be v x d")
    if targets.shape != x.shape[:-1]:
        raise ValueError("targets must have x's leading dimensions")
    t = _tokens(targets, w.nrows, "targets")
    dev = x.get_device()
    _same_device(dev, weight, "weight")
    _same_device(dev, targets, "targets")
    return a, w, t


@_on_device(0, "x")
def linear_cross_entropy(x, weight, targets, scale=1.0):
    """(loss, lse), float32, one per row of ``x``: with the logits ``z = scale * x
    @ weight.T`` over the rows of ``weight`` (v x d), lse = log sum exp z and loss
    = lse - z[target]  (spsyrk_linear_cross_entropy).  The logits are formed piece
    by piece and not kept.  ``targets``: int32 or int64 of x's leading dimensions;
    outside [0, v) they are padding, with loss 0."""
    lib = _sp._lib or _sp.library()
    _unrecorded("linear_cross_entropy_grad", x, weight)
    a, w, t = _linear(x, weight, targets)
    loss = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    lse = torch.empty_like(loss)
    arena = _arena(x.get_device())
    _check(lib.spsyrk_linear_cross_entropy(_byref(a), _byref(w), _byref(t), scale, _byref(arena.struct),
                                           _raw_stream(x.get_device()), loss.data_ptr(), lse.data_ptr()), arena)
    return loss, lse


@_on_device(0, "x")
def linear_cross_entropy_grad(x, weight, targets, scale=1.0, row_weight=None):
    """(loss, dx, dweight): ``linear_cross_entropy`` together with the gradients,
    of the inputs' types, of ``(row_weight * loss).sum()`` (``row_weight``:
    float32, one per row; None for ones)  (spsyrk_linear_cross_entropy_grad).
    Padding and rows of weight 0 take no part, whatever x holds there."""
    lib = _sp._lib or _sp.library()
    a, w, t = _linear(x, weight, targets)
    wp = _vector(row_weight, "row_weight", a.nrows, (torch.float32,), x.get_device())
    loss = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    dx, dw = _like(x), _like(weight)
    ox = _sp._Dense(a.nrows, a.ncols, a.ncols, a.dtype, dx.data_ptr())
    ow = _sp._Dense(w.nrows, w.ncols, w.ncols, w.dtype, dw.data_ptr())
    arena = _arena(x.get_device())
    _check(lib.spsyrk_linear_cross_entropy_grad(_byref(a), _byref(w), _byref(t), scale, wp, _byref(arena.struct),
                                                _raw_stream(x.get_device()), loss.data_ptr(), _byref(ox),
                                                _byref(ow)), arena)
    return loss, dx, dw
