"""Operators of a model whose inputs and targets are sparse rows: table lookup,
layer norm and distillation, forward and backward (C-ABI in
``include/spsyrk.h``).

Dense arguments are torch tensors of one GPU, float32, float16 or bfloat16,
whose last dimension is contiguous; rows may be strided (a slice of columns).
Leading dimensions count as rows where they can be walked with one stride.
Work is enqueued on the current stream of the tensors' device and nothing waits
for it.  Autograd does not record these calls: every gradient is a call of its
own.  ``embed``, ``layer_norm`` and ``distill`` refuse inputs that require a
gradient while gradients are recorded, as it would be lost; call them under
``torch.no_grad()`` or on detached tensors.
"""
from __future__ import annotations

import ctypes
import functools
import threading

import torch

import paper_2608_09713_amd as _sp

_DTYPE = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_byref = ctypes.byref


def _rows(t, name):
    """_Dense of the tensor's rows; the last dimension is the columns."""
    dt = _DTYPE.get(t.dtype)
    if dt is None:
        raise TypeError(f"{name} must be float32, float16 or bfloat16, not {t.dtype}")
    if not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.dim() < 1:
        raise ValueError(f"{name} must have at least one dimension")
    cols = t.shape[-1]
    if t.is_contiguous():
        rows = t.numel() // cols if cols else t.shape[:-1].numel()
        return _sp._Dense(rows, cols, cols, dt, t.data_ptr())
    try:
        v = t.view(-1, cols) if t.dim() != 2 else t
    except RuntimeError:
        v = None
    if v is None or (cols > 1 and v.stride(1) != 1) or (v.shape[0] > 1 and v.stride(0) < cols):
        raise ValueError(f"{name} must have rows of contiguous elements at one stride")
    return _sp._Dense(v.shape[0], cols, max(v.stride(0), cols), dt, v.data_ptr())


def _unrecorded(gradient, *tensors):
    """Refuses inputs whose gradient autograd would be expected to pass on."""
    for t in tensors:
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise RuntimeError("autograd does not record this call, and an input requires a gradient: call it under "
                               f"torch.no_grad() or on detached tensors, and take the gradient from {gradient}")


def _like(t):
    """A contiguous tensor of t's shape and type."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _vector(t, name, n, dtypes, device):
    """Address of a contiguous vector of n elements (None: null)."""
    if t is None:
        return None
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(map(str, dtypes))}, not {t.dtype}")
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous, of {n} elements")
    _same_device(device, t, name)
    return t.data_ptr()


def _same_device(device, t, name):
    """device: an index, as get_device gives (-1: the host)."""
    if t.get_device() != device:
        raise ValueError(f"{name} must be on device {device}, not on {t.device}")


def _entries_csr(A, values, name):
    """_Entries of a DeviceCSR."""
    for t, want in ((A.row_ptr, (torch.int64,)), (A.col_idx, (torch.int32, torch.int64))):
        if t.dtype not in want:
            raise TypeError(f"{name}: row_ptr must be int64, col_idx int32 or int64")
        if not t.is_cuda or not t.is_contiguous():
            raise TypeError(f"{name}: CSR arrays must be contiguous device tensors")
    if A.row_ptr.numel() != A.nrows + 1 or A.col_idx.numel() < A.nnz:
        raise ValueError(f"{name}: row_ptr must have nrows + 1 entries and col_idx at least nnz")
    v, vp, vt = A.values, None, 0
    if v is not None:
        vt = _DTYPE.get(v.dtype)
        if vt is None:
            raise TypeError(f"{name}: values must be float32, float16 or bfloat16, not {v.dtype}")
        if v.numel() < A.nnz or not v.is_contiguous():
            raise ValueError(f"{name}: values must be contiguous, of at least nnz entries")
        _same_device(A.row_ptr.get_device(), v, f"{name}.values")
        vp = v.data_ptr()
    elif values:
        raise TypeError(f"{name}: values are required")
    _same_device(A.row_ptr.get_device(), A.col_idx, f"{name}.col_idx")
    return _sp._Entries(A.nrows, A.ncols, A.nnz, A.row_ptr.data_ptr(), 0, 0, 0, A.col_idx.data_ptr(),
                        A.col_idx.element_size(), vt, vp)


def _tokens(t, ncols, name):
    """_Entries of a tensor of tokens, one row each."""
    if t.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"{name} must be a DeviceCSR, or int32 or int64 tokens, not {t.dtype}")
    if not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    n, stride = t.numel(), 1
    if not t.is_contiguous():
        if t.dim() != 1 or t.stride(0) < 0:
            raise ValueError(f"{name} must be contiguous, or one strided dimension")
        stride = t.stride(0)
    return _sp._Entries(n, ncols, 0, None, 1, stride, 0, t.data_ptr(), t.element_size(), 0, None)


_local = threading.local()
# (the handle and the index alone: a Stream object costs 2 us of a call)
_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice


def _arena(device):
    """This thread's allocator for the device of an index (its callbacks are made
    once; it holds nothing between calls)."""
    arenas = getattr(_local, "arenas", None)
    if arenas is None:
        arenas = _local.arenas = {}
    arena = arenas.get(device)
    if arena is None:
        arena = arenas[device] = _sp._TorchArena(torch.device("cuda", device))
    return arena


def _on_device(position, name):
    """Decorator: the device of the named dense argument is the current one
    during the call."""
    def decorate(fn):
        @functools.wraps(fn)
        def call(*args, **kwargs):
            t = args[position] if len(args) > position else kwargs.get(name)
            if isinstance(t, torch.Tensor) and t.is_cuda and t.get_device() != _current_device():
                with torch.cuda.device(t.device):
                    return fn(*args, **kwargs)
            return fn(*args, **kwargs)
        return call
    return decorate


def _check(rc, arena=None):
    if rc != 0:
        raise _sp.SpsyrkError(rc, _sp.library().spsyrk_last_error_detail().decode())
    if arena is not None and arena.live:
        arena.live.clear()
        raise RuntimeError("library left allocations unreleased")


@_on_device(1, "weight")
def embed(rows, weight, scale=1.0):
    """Rows of the table ``weight`` (v x d): ``scale`` times ``weight[token]`` for
    a tensor of tokens (shape + (d,); zeros for tokens outside [0, v), which are
    padding), or ``scale * A @ weight`` for a DeviceCSR (m x d; its values, or
    ones, weight the entries)  (spsyrk_embed)."""
    lib = _sp._lib or _sp.library()
    _unrecorded("embed_grad", weight, None if isinstance(rows, torch.Tensor) else rows.values)
    w = _rows(weight, "weight")
    if weight.dim() != 2:
        raise ValueError("weight must be v x d")
    dev = weight.get_device()
    if isinstance(rows, torch.Tensor):
        a, csr, shape = _tokens(rows, w.nrows, "rows"), False, rows.shape
        _same_device(dev, rows, "rows")
    else:
        a, csr, shape = _entries_csr(rows, False, "rows"), True, (rows.nrows,)
        _same_device(dev, rows.row_ptr, "rows")
    out = torch.empty((*shape, w.ncols), dtype=weight.dtype, device=weight.device)
    y = _sp._Dense(a.nrows, w.ncols, w.ncols, w.dtype, out.data_ptr())
    arena = _arena(dev) if csr else None
    _check(lib.spsyrk_embed(_byref(a), _byref(w), scale, _byref(arena.struct) if csr else None,
                            _raw_stream(dev), _byref(y)), arena)
    return out


@_on_device(1, "grad")
def embed_grad(rows, grad, v, scale=1.0):
    """The gradient (v x d) of the table looked up by ``embed(rows, weight,
    scale)`` for the gradient ``grad`` of its result: ``scale * A.T @ grad``,
    summed by entries sorted by column (spsyrk_embed_grad)."""
    lib = _sp._lib or _sp.library()
    g, dev = _rows(grad, "grad"), grad.get_device()
    if isinstance(rows, torch.Tensor):
        a, first = _tokens(rows, v, "rows"), rows
    else:
        a, first = _entries_csr(rows, False, "rows"), rows.row_ptr
    _same_device(dev, first, "rows")
    out = torch.empty((v, g.ncols), dtype=grad.dtype, device=grad.device)
    w = _sp._Dense(v, g.ncols, g.ncols, g.dtype, out.data_ptr())
    arena = _arena(dev)
    _check(lib.spsyrk_embed_grad(_byref(a), _byref(g), scale, _byref(arena.struct), _raw_stream(dev),
                                 _byref(w)), arena)
    return out


def _params(x, d, weight, bias, what):
    """(type code, addresses) of the layer norm's parameters."""
    first = weight if weight is not None else bias
    pt = x.dtype if first is None else first.dtype
    if pt not in (torch.float32, x.dtype):
        raise TypeError(f"{what}: weight and bias must be float32 or {x.dtype}, not {pt}")
    return (_DTYPE[pt], _vector(weight, "weight", d, (pt,), x.get_device()),
            _vector(bias, "bias", d, (pt,), x.get_device()))


@_on_device(0, "x")
def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """(y, mean, rstd): y = (x - mean) rstd weight + bias over the last dimension,
    with the rows' mean and 1 / sqrt(var + eps) as float32 (spsyrk_layer_norm).
    ``weight`` and ``bias``: float32 or x's type, None for ones and zeros."""
    lib = _sp._lib or _sp.library()
    _unrecorded("layer_norm_grad", x, weight, bias)
    a = _rows(x, "x")
    pt, wp, bp = _params(x, a.ncols, weight, bias, "layer_norm")
    y = _like(x)
    mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    rstd = torch.empty_like(mean)
    o = _sp._Dense(a.nrows, a.ncols, a.ncols, a.dtype, y.data_ptr())
    _check(lib.spsyrk_layer_norm(_byref(a), wp, bp, pt, eps, _raw_stream(x.get_device()), _byref(o),
                                 mean.data_ptr(), rstd.data_ptr()))
    return y, mean, rstd


@_on_device(0, "grad")
def layer_norm_grad(grad, x, mean, rstd, weight=None, bias=None):
    """(dx, dweight, dbias) of ``layer_norm(x, weight, bias)`` for the gradient
    ``grad`` of y; dweight and dbias have the parameters' type and are None for
    a parameter that is None (spsyrk_layer_norm_grad)."""
    lib = _sp._lib or _sp.library()
    g, a = _rows(grad, "grad"), _rows(x, "x")
    if grad.shape != x.shape:
        raise ValueError("grad and x must have one shape")
    _same_device(x.get_device(), grad, "grad")
    pt, wp, _ = _params(x, a.ncols, weight, bias, "layer_norm_grad")
    mp = _vector(mean, "mean", a.nrows, (torch.float32,), x.get_device())
    rp = _vector(rstd, "rstd", a.nrows, (torch.float32,), x.get_device())
    dx = _like(x)
    dw = None if weight is None else torch.empty_like(weight)
    db = None if bias is None else torch.empty_like(bias)
    o = _sp._Dense(a.nrows, a.ncols, a.ncols, a.dtype, dx.data_ptr())
    arena = _arena(x.get_device())
    _check(lib.spsyrk_layer_norm_grad(_byref(g), _byref(a), mp, rp, wp, pt, _byref(arena.struct),
                                      _raw_stream(x.get_device()), _byref(o),
                                      None if dw is None else dw.data_ptr(), None if db is None else db.data_ptr()),
           arena)
    return dx, dw, db


def _teacher(teacher, s, logits):
    """_Entries of a DeviceCSR, or of a (values, indices) pair with the logits' leading dimensions."""
    if not isinstance(teacher, tuple):
        e = _entries_csr(teacher, True, "teacher")
        _same_device(logits.get_device(), teacher.row_ptr, "teacher")
        return e
    values, indices = teacher
    if values.shape != indices.shape or values.shape[:-1] != logits.shape[:-1]:
        raise ValueError("the teacher's values and indices must have one shape, and the logits' leading dimensions")
    if indices.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"the teacher's indices must be int32 or int64, not {indices.dtype}")
    _same_device(logits.get_device(), values, "teacher values")
    _same_device(logits.get_device(), indices, "teacher indices")
    v = _rows(values, "teacher values")
    k = v.ncols
    stride = k
    if not indices.is_contiguous():
        if indices.dim() != 2 or (k > 1 and indices.stride(1) != 1):
            raise ValueError("the teacher's indices must be contiguous, or strided rows of contiguous elements")
        stride = indices.stride(0)
    return _sp._Entries(s.nrows, s.ncols, 0, None, k, stride, v.ld, indices.data_ptr(), indices.element_size(),
                        v.dtype, values.data_ptr())


@_on_device(0, "logits")
def distill(logits, teacher, temperature=1.0):
    """Loss (float32, one per row of ``logits``) of distilling the teacher's
    stored entries: temperature^2 times the divergence of the logits' softmax
    from the teacher's softmax over the row's entries (spsyrk_distill).
    ``teacher``: a DeviceCSR over the logits' columns, or a tuple (values,
    indices) as torch.topk returns; indices outside the columns are padding."""
    lib = _sp._lib or _sp.library()
    _unrecorded("distill_grad", logits, teacher[0] if isinstance(teacher, tuple) else teacher.values)
    s = _rows(logits, "logits")
    t = _teacher(teacher, s, logits)
    loss = torch.empty(logits.shape[:-1], dtype=torch.float32, device=logits.device)
    arena = _arena(logits.get_device())
    _check(lib.spsyrk_distill(_byref(s), _byref(t), temperature, _byref(arena.struct),
                              _raw_stream(logits.get_device()), loss.data_ptr()), arena)
    return loss


@_on_device(0, "logits")
def distill_grad(logits, teacher, temperature=1.0, weight=None):
    """(loss, gradient): ``distill`` together with the gradient, of the logits'
    type, of ``(weight * loss).sum()`` (``weight``: float32, one per row; None
    for ones)  (spsyrk_distill_grad)."""
    lib = _sp._lib or _sp.library()
    s = _rows(logits, "logits")
    t = _teacher(teacher, s, logits)
    wp = _vector(weight, "weight", s.nrows, (torch.float32,), logits.get_device())
    loss = torch.empty(logits.shape[:-1], dtype=torch.float32, device=logits.device)
    grad = _like(logits)
    g = _sp._Dense(s.nrows, s.ncols, s.ncols, s.dtype, grad.data_ptr())
    arena = _arena(logits.get_device())
    _check(lib.spsyrk_distill_grad(_byref(s), _byref(t), temperature, wp, _byref(arena.struct),
                                   _raw_stream(logits.get_device()), loss.data_ptr(), _byref(g)), arena)
    return loss, grad
