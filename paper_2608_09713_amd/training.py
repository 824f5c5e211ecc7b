"""Operators of a training step: the cross entropy of a linear layer over many
columns and the norms around a block, forward and backward, and an AdamW step
over many tensors (C-ABI in ``include/spsyrk.h``).

What ``rows.py`` says of tensors, streams and autograd holds here too: dense
arguments are float32, float16 or bfloat16 rows of one GPU, work is enqueued on
the current stream, gradients are calls of their own, and a forward call refuses
an input whose gradient would be lost.
"""
from __future__ import annotations

import ctypes
import itertools
import operator
import struct
from typing import NamedTuple, Optional

import torch

import paper_2608_09713_amd as _sp

from .rows import (_DTYPE, _arena, _byref, _check, _like, _on_device, _raw_stream, _rows, _same_device, _tokens,
                   _unrecorded, _vector)


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


def _block_params(x, d, post, pre, what):
    """(type code, addresses) of the norms' weights."""
    first = post if post is not None else pre
    pt = x.dtype if first is None else first.dtype
    if pt not in (torch.float32, x.dtype):
        raise TypeError(f"{what}: post and pre must be float32 or {x.dtype}, not {pt}")
    dev = x.get_device()
    return _DTYPE[pt], _vector(post, "post", d, (pt,), dev), _vector(pre, "pre", d, (pt,), dev)


def _gate(x, gate):
    """_Dense of a gate (None: null)."""
    if gate is None:
        return None
    g = _rows(gate, "gate")
    if gate.dtype not in (torch.float32, x.dtype):
        raise TypeError(f"gate must be float32 or {x.dtype}, not {gate.dtype}")
    _same_device(x.get_device(), gate, "gate")
    return g


def _same_rows(x, t, name):
    if t.shape != x.shape or t.dtype != x.dtype:
        raise ValueError(f"{name} must have the shape and type {tuple(x.shape)}, {x.dtype}")
    _same_device(x.get_device(), t, name)
    return _rows(t, name)


def _ref(x):
    return None if x is None else _byref(x)


@_on_device(0, "x")
def block_norm(x, block, gate=None, scale=1.0, post=None, pre=None, norm_block=True, eps=1e-6):
    """(y, h, rstd_post, rstd_pre) over the last dimension: u = block times
    1 / sqrt(mean block^2 + eps) times ``post`` (``norm_block`` false: u = block,
    and rstd_post is None); y = x + scale * gate * u; h = y / sqrt(mean y^2 + eps)
    * ``pre``  (spsyrk_block_norm).  ``post``, ``pre``: float32 or x's type, None
    for ones.  ``gate``: float32 or x's type, (d,), or (..., d) with rows that
    divide x's: each holds for as many consecutive rows; None for ones."""
    lib = _sp._lib or _sp.library()
    _unrecorded("block_norm_grad", x, block, gate, post, pre)
    a = _rows(x, "x")
    b = _same_rows(x, block, "block")
    g = _gate(x, gate)
    pt, pp, qp = _block_params(x, a.ncols, post, pre, "block_norm")
    dev = x.get_device()
    y, h = _like(x), _like(x)
    rstd_pre = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    rstd_post = torch.empty_like(rstd_pre) if norm_block else None
    oy = _sp._Dense(a.nrows, a.ncols, a.ncols, a.dtype, y.data_ptr())
    oh = _sp._Dense(a.nrows, a.ncols, a.ncols, a.dtype, h.data_ptr())
    _check(lib.spsyrk_block_norm(_byref(a), _byref(b), _ref(g), scale, pp, qp, pt, not norm_block, eps,
                                 _raw_stream(dev), _byref(oy), _byref(oh),
                                 None if rstd_post is None else rstd_post.data_ptr(), rstd_pre.data_ptr()))
    return y, h, rstd_post, rstd_pre


@_on_device(1, "dh")
def block_norm_grad(dy, dh, y, block, rstd_post, rstd_pre, gate=None, scale=1.0, post=None, pre=None):
    """(dx, dblock, dgate, dpost, dpre) of ``block_norm`` for the gradients ``dy``
    (None: none) of y and ``dh`` of h, with its y, rstd_post (None: the block was
    not normed) and rstd_pre; dgate, dpost and dpre have their arguments' types and
    shapes and are None where those are  (spsyrk_block_norm_grad)."""
    lib = _sp._lib or _sp.library()
    e = _rows(dh, "dh")
    a = _same_rows(dh, y, "y")
    b = _same_rows(dh, block, "block")
    f = None if dy is None else _same_rows(dh, dy, "dy")
    g = _gate(y, gate)
    pt, pp, qp = _block_params(y, a.ncols, post, pre, "block_norm_grad")
    dev = dh.get_device()
    r1 = _vector(rstd_post, "rstd_post", a.nrows, (torch.float32,), dev)
    r2 = _vector(rstd_pre, "rstd_pre", a.nrows, (torch.float32,), dev)
    if post is not None and rstd_post is None:
        raise ValueError("a block without a norm has no weights of one: post must be None")
    dx, db = _like(y), _like(y)
    dgate = None if gate is None else _like(gate)
    dpost = None if post is None else torch.empty_like(post)
    dpre = None if pre is None else torch.empty_like(pre)
    ox = _sp._Dense(a.nrows, a.ncols, a.ncols, a.dtype, dx.data_ptr())
    ob = _sp._Dense(a.nrows, a.ncols, a.ncols, a.dtype, db.data_ptr())
    og = None if g is None else _sp._Dense(g.nrows, g.ncols, g.ncols, g.dtype, dgate.data_ptr())
    arena = _arena(dev)
    _check(lib.spsyrk_block_norm_grad(_ref(f), _byref(e), _byref(a), _byref(b), r1, r2, _ref(g), scale, pp, qp, pt,
                                      _byref(arena.struct), _raw_stream(dev), _byref(ox), _byref(ob), _ref(og),
                                      None if dpost is None else dpost.data_ptr(),
                                      None if dpre is None else dpre.data_ptr()), arena)
    return dx, db, dgate, dpost, dpre


ADAM_BLOCK = 256  # elements that share a scale in 8-bit states


class AdamState(NamedTuple):
    """A tensor's states: m and v in float32, or codes (int8 and uint8) with a
    float32 scale for every 256 elements."""
    m: torch.Tensor
    v: torch.Tensor
    m_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None


def adam_state(param, bits=32):
    """States of zeros for ``param``, of 32 or 8 bits per element."""
    if bits == 32:
        return AdamState(torch.zeros(param.shape, dtype=torch.float32, device=param.device),
                         torch.zeros(param.shape, dtype=torch.float32, device=param.device))
    if bits != 8:
        raise ValueError("states have 32 or 8 bits")
    blocks = -(-param.numel() // ADAM_BLOCK)
    return AdamState(torch.zeros(param.shape, dtype=torch.int8, device=param.device),
                     torch.zeros(param.shape, dtype=torch.uint8, device=param.device),
                     torch.zeros(blocks, dtype=torch.float32, device=param.device),
                     torch.zeros(blocks, dtype=torch.float32, device=param.device))


def _state_bits(state, numel):
    """8 or 32; checks a state's types and sizes."""
    m, v, ms, vs = state
    if m.dtype == torch.float32 and v.dtype == torch.float32 and ms is None and vs is None:
        bits = 32
    elif (m.dtype == torch.int8 and v.dtype == torch.uint8 and ms is not None and vs is not None
          and ms.dtype == torch.float32 and vs.dtype == torch.float32):
        bits = 8
        if ms.numel() != -(-numel // ADAM_BLOCK) or vs.numel() != ms.numel():
            raise ValueError(f"m_scale and v_scale must have one element for every {ADAM_BLOCK} of the tensor")
    else:
        raise TypeError("a state must be two float32 tensors, or int8 and uint8 codes with float32 scales")
    if m.numel() != numel or v.numel() != numel:
        raise ValueError("a state must have the tensor's size")
    return bits


_ptr = torch.Tensor.data_ptr
_tensors = None


def _native():
    """The module of csrc/tensors.cpp; raises if that has not been built."""
    global _tensors
    if _tensors is None:
        try:
            from . import _tensors as module
        except ImportError as e:
            raise ImportError("_tensors.so is missing or of another torch: run `python -m paper_2608_09713_amd.build` "
                              "(or __graft_entry__.build()) first") from e
        _tensors = module
    return _tensors


class AdamWPlan:
    """AdamW steps over the same tensors.  The plan keeps the tensors; their
    addresses, sizes, types and layouts are read again at every step, so it follows
    tensors whose storage was exchanged (``.data = ...``) for one of the same type and
    size, and refuses others.  A gradient that was its parameter's ``grad`` has to stay
    that (``zero_grad(set_to_none=False)``).  A step counts as a change in place of all
    that it writes, so that autograd refuses a backward pass that saved it before."""

    def __init__(self, params, grads, states, masters=None):
        params, grads = list(params), list(grads)
        states = [s if isinstance(s, AdamState) else AdamState(*s) for s in states]
        masters = None if masters is None else list(masters)
        if not len(params) == len(grads) == len(states) or (masters is not None and len(masters) != len(params)):
            raise ValueError("params, grads, states and masters must have one length")
        self.params, self.grads, self.states, self.masters = params, grads, states, masters
        self._device = params[0].get_device() if params else -1
        if params and not params[0].is_cuda:
            raise TypeError("params must be device tensors")
        self._of_autograd = [(p, g) for p, g in zip(params, grads) if p.is_leaf and p.grad is g]
        columns = [params, masters or [], *([s[c] for s in states] for c in range(4)), grads]
        # (param, master, m, v, m_scale, v_scale, grad: those that there are)
        self._columns = [c for c, column in enumerate(columns) if any(t is not None for t in column)]
        self._all = tuple(t for c in self._columns for t in columns[c])
        self._written = self._all[:len(self._all) - len(grads)]
        notes = _native().note(self._all)
        self._kinds = self._checked(notes)
        groups = {}
        for k, kind in enumerate(self._kinds):
            groups.setdefault(kind[1:], []).append(k)
        # (one call for each kind of tensor)
        self._calls = [(_sp._AdamStep(_DTYPE[pt], _DTYPE[gt], bits), (_sp._AdamTensor * len(index))(), index)
                       for (pt, gt, bits, _), index in groups.items()]
        self._fill(notes)

    def _checked(self, notes):
        """(size, parameter's type, gradient's type, state's bits, with a master copy) of every tensor."""
        words = memoryview(notes).cast("q").tolist()
        here = (1 << 16) + (self._device & 0xffff)  # contiguous, on the device
        if {made >> 32 for made in words[2::3]} - {-1, here} or not all(map(operator.ge, words[0::3], map(bool, words[1::3]))):
            for t in self._all:
                if t is not None:
                    if t.get_device() != self._device:
                        raise ValueError("all tensors must be on one device")
                    if not t.is_contiguous():
                        raise ValueError("all tensors must be contiguous")
                    if t.numel() and not t.data_ptr():
                        raise ValueError("a tensor of the plan has no storage")
        kinds = []
        for k, (p, g, s) in enumerate(zip(self.params, self.grads, self.states)):
            w = None if self.masters is None else self.masters[k]
            if p.dtype not in _DTYPE:
                raise TypeError(f"params must be float32, float16 or bfloat16, not {p.dtype}")
            if g is None:
                raise TypeError("every parameter must have a gradient, not None")
            if g.dtype not in (torch.float32, p.dtype):
                raise TypeError(f"grads must be float32 or the parameter's type, not {g.dtype}")
            n = p.numel()
            if g.numel() != n:
                raise ValueError("a gradient must have its parameter's size")
            if w is not None:
                if p.dtype == torch.float32:
                    raise TypeError("float32 parameters have no master copy")
                if w.dtype != torch.float32 or w.numel() != n:
                    raise TypeError("a master copy must be float32, of its parameter's size")
            kinds.append((n, p.dtype, g.dtype, _state_bits(s, n), w is not None))
        return kinds

    def _follow(self):
        """The tensors' present addresses into the tables.  What a step relies on is
        compared whole: a tensor that has changed its size, type or order may still
        have its old address."""
        for p, g in self._of_autograd:
            if p.grad is not g:
                raise ValueError("a parameter's grad is no longer the tensor that the plan was given (set to None and made "
                                 "anew?): keep it, or make a plan of the new ones")
        notes = _tensors.note(self._all)
        if notes == self._seen:
            return
        if self._checked(notes) != self._kinds:
            raise ValueError("a tensor of the plan has changed its type or size")
        self._fill(notes)

    def _fill(self, notes):
        words, n = memoryview(notes).cast("q").tolist(), len(self.params)
        at, size = words[0::3], words[1::3]
        self._distinct(at, size)
        columns = [[0] * n] * 7
        for i, c in enumerate(self._columns):
            columns[c] = at[i * n:i * n + n]
        param, master, m, v, m_scale, v_scale, grad = columns
        rows = list(zip((k[0] for k in self._kinds), param, grad, master, m, v, m_scale, v_scale))
        for _, table, index in self._calls:
            struct.pack_into(f"{8 * len(index)}q", table, 0, *itertools.chain.from_iterable(rows[k] for k in index))
        self._seen = notes

    def _distinct(self, at, size):
        """Refuses tensors that are written twice in a step, or read as a gradient
        while they are written (but for a parameter that is its own gradient, each
        element of which is read and written by one thread)."""
        ends = list(map(operator.add, at, size))
        spans = sorted(zip(at, ends))
        if not any(map(operator.gt, (end for _, end in spans), (start for start, _ in spans[1:]))):
            return  # (no two lie across each other)
        n, written = len(self.params), len(self._written)
        own = {written + k for k in range(n) if at[k] == at[written + k] and self.grads[k].dtype == self.params[k].dtype}
        last = {True: 0, False: 0}  # where what was written (read) so far ends
        for start, end, write in sorted((at[k], ends[k], k < written) for k in range(len(at)) if size[k] and k not in own):
            if start < last[True] or (write and start < last[False]):
                raise ValueError("tensors that a step writes must not overlap, nor be the gradients of others (the same "
                                 "one twice?)")
            last[write] = max(last[write], end)

    def step(self, lr, step, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, grad_scale=None):
        """One step, in place (``adamw``)."""
        if not self._calls:
            return
        scale = None
        if grad_scale is not None:
            scale = _vector(grad_scale, "grad_scale", 1, (torch.float32,), self._device)
        lib = _sp._lib or _sp.library()
        self._follow()
        with torch.cuda.device(self._device):
            for how, table, _ in self._calls:
                how.step, how.lr, how.eps, how.weight_decay, how.grad_scale = step, lr, eps, weight_decay, scale
                how.beta1, how.beta2 = betas
                _check(lib.spsyrk_adamw(table, len(table), _byref(how), _raw_stream(self._device)))
        _tensors.changed(self._written)


def adamw_plan(params, grads, states, masters=None):
    """An ``AdamWPlan``, for many steps over the same tensors: ``plan.step(lr,
    step, betas, eps, weight_decay, grad_scale)`` is ``adamw`` over them."""
    return AdamWPlan(params, grads, states, masters)


def adamw(params, grads, states, lr, step, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, grad_scale=None,
          masters=None):
    """One AdamW step over many tensors, in place  (spsyrk_adamw): ``states`` from
    ``adam_state``, one for each parameter; ``step`` counts from 1; ``grads`` of
    float32 or the parameters' type, times ``grad_scale`` (a float32 device tensor
    of one element) if given; ``masters``: float32 copies of 16-bit parameters,
    which are stepped and rounded into them (None for a parameter without one).
    The rates are taken at the call: a captured call repeats them."""
    AdamWPlan(params, grads, states, masters).step(lr, step, betas, eps, weight_decay, grad_scale)


def adam_values(states):
    """[(m, v)] in float32 of every state (the tensors themselves for states of 32
    bits)  (spsyrk_adam_values)."""
    states = list(states)
    out, narrow = [], []
    for s in states:
        if _state_bits(s, s[0].numel()) == 32:
            out.append((s[0], s[1]))
            continue
        for t in s:
            if not t.is_cuda:
                raise TypeError("states must be device tensors")
            if not t.is_contiguous():
                raise ValueError("states must be contiguous")
            _same_device(s[0].get_device(), t, "a state's tensor")
        _same_device((narrow[0][0] if narrow else s)[0].get_device(), s[0], "a state")
        out.append((torch.empty(s[0].shape, dtype=torch.float32, device=s[0].device),
                    torch.empty(s[1].shape, dtype=torch.float32, device=s[1].device)))
        narrow.append((s, out[-1]))
    if narrow:
        lib = _sp._lib or _sp.library()
        dev = narrow[0][0][0].get_device()
        table = (_sp._AdamTensor * len(narrow))()
        for row, (s, _) in zip(table, narrow):
            row.n, row.m, row.v, row.m_scale, row.v_scale = s[0].numel(), *map(_ptr, s)
        ms, vs = ((ctypes.c_void_p * len(narrow))(*(o[k].data_ptr() for _, o in narrow)) for k in (0, 1))
        with torch.cuda.device(dev):
            _check(lib.spsyrk_adam_values(table, len(table), ms, vs, _raw_stream(dev)))
    return out
