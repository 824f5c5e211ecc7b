"""What an AdamW plan sees of its tensors before a step, on the host: tensors of
the host stand in for a device's, and no step is enqueued."""
import ctypes
import os

import pytest
import torch

import paper_2608_09713_amd as sp
from paper_2608_09713_amd import build
from tests.test_rows_refusals import INVALID, P, lib  # noqa: F401
from tests.test_training_refusals import adam


@pytest.fixture(scope="module", autouse=True)
def _tensors():
    if not os.path.exists(build.TENSORS):
        build.build_tensors()


class OnDevice(torch.Tensor):
    is_cuda = True


def host(t):
    return t.as_subclass(OnDevice)


def plan_of(*shapes, bits=32, dtype=torch.float32):
    params = [host(torch.zeros(s, dtype=dtype)) for s in shapes]
    grads = [torch.ones(s, dtype=dtype) for s in shapes]
    return sp.adamw_plan(params, grads, [sp.adam_state(p, bits) for p in params]), params, grads


@pytest.mark.parametrize("which", ["param", "grad", "m", "v"])
@pytest.mark.parametrize("change", [lambda t: t[:32], lambda t: t.t(), lambda t: t.view(torch.int32), lambda t: t[:0],
                                    lambda t: t[:, :1]], ids=["half", "turned", "type", "empty", "column"])
def test_a_change_at_the_same_address_is_refused(which, change):
    plan, params, grads = plan_of((64, 64), (5,))
    t = dict(param=params[0], grad=grads[0], m=plan.states[0].m, v=plan.states[0].v)[which]
    whole, at = t.data, t.data_ptr()
    t.data = change(whole)
    assert t.data_ptr() in (at, 0)
    for _ in range(2):  # (and stays refused)
        with pytest.raises((ValueError, TypeError)):
            plan._follow()
    t.data = whole
    plan._follow()


def test_a_scale_that_lost_elements_is_refused():
    plan, _, _ = plan_of((600,), bits=8)
    s = plan.states[0].m_scale
    s.data = s.data[:1]
    with pytest.raises(ValueError, match="m_scale"):
        plan._follow()


def test_another_shape_of_the_same_elements_is_followed():
    plan, params, grads = plan_of((6, 4), (3,))
    params[0].data = params[0].data.view(24)
    grads[0].data = torch.full((24,), 2.0)
    plan._follow()
    table = plan._calls[0][1]
    assert table[0].n == 24 and table[0].param == params[0].data_ptr() and table[0].grad == grads[0].data_ptr()
    assert table[1].grad == grads[1].data_ptr()


def test_the_binding_says_what_is_not_built(monkeypatch):
    import sys

    from paper_2608_09713_amd import training
    monkeypatch.setattr(training, "_tensors", None)
    monkeypatch.setitem(sys.modules, "paper_2608_09713_amd._tensors", None)
    monkeypatch.delattr(sp, "_tensors", raising=False)
    with pytest.raises(ImportError, match="build"):
        plan_of((4,))


def test_notes_are_of_tensors():
    from paper_2608_09713_amd import training
    note = training._native().note
    t = torch.zeros(6)
    assert note((t, t[1:])) == note((t, t[1:])) != note((t, t[2:]))
    assert note(()) == b"" and len(note((t,))) * 2 == len(note((t, None))) and note((None,)) != note((t,))
    for bad in ([t], None, (3,)):
        with pytest.raises(TypeError):
            note(bad)


@pytest.mark.parametrize("order", [1, -1])
def test_copies_of_some_parameters(order):
    # (32-bit parameters have no copy: None beside the others')
    shapes, types = [(300,), (7,), (40,)], [torch.bfloat16, torch.float32, torch.float16]
    params = [host(torch.zeros(s, dtype=t)) for s, t in zip(shapes, types)][::order]
    masters = [None if p.dtype == torch.float32 else p.float() for p in params]
    plan = sp.adamw_plan(params, [torch.ones_like(p) for p in params], [sp.adam_state(p) for p in params], masters)
    assert len(plan._calls) == 3
    for how, table, _ in plan._calls:
        row, k = table[0], next(k for k, p in enumerate(params) if p.numel() == table[0].n)
        assert row.master == (None if masters[k] is None else masters[k].data_ptr())
    twice = [params[0], params[0]]
    with pytest.raises(ValueError, match="overlap"):
        sp.adamw_plan(params[:1] + [host(torch.zeros_like(params[0]))], twice, [sp.adam_state(p) for p in twice],
                      [masters[0], masters[0]])


def test_an_empty_tensor_in_front(lib):  # noqa: F811
    # (its address, and its copy's, may be null: the others decide whether copies are given)
    def step(*tensors, pt=2):
        table = (sp._AdamTensor * len(tensors))(*tensors)
        how = sp._AdamStep(pt, pt, 32, 1, 1e-3, 0.9, 0.99, 1e-8, 0.1, None)
        return lib.spsyrk_adamw(table, len(tensors), ctypes.byref(how), None)

    empty = adam(n=0, param=None, grad=None, m=None, v=None)
    mixed = (adam(master=P), adam())
    assert step(empty, *mixed) == step(*mixed) == step(*mixed[::-1]) == INVALID
    assert b"all tensors or for none" in lib.spsyrk_last_error_detail()
    # (an address off its boundary is refused behind that check, before any device call)
    assert step(empty, adam(master=P + 2)) == step(empty, adam(master=P), adam(master=P + 2)) == INVALID
    assert b"master is not aligned" in lib.spsyrk_last_error_detail()
    assert step(empty, adam(master=P), pt=0) == INVALID
    assert b"no master copy" in lib.spsyrk_last_error_detail()


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_that_a_step_writes_are_refused(bits):
    # (a gradient is read while other tensors, or other elements of the same one, are written)
    a, b, g = host(torch.zeros(512)), host(torch.zeros(512)), torch.ones(512)
    s, r = sp.adam_state(a, bits), sp.adam_state(b, bits)
    buffer = torch.zeros(1024)
    for params, grads in (([a, b], [g, a]), ([a, b], [b, g]), ([host(buffer[:512])], [buffer[100:612]]),
                          ([host(buffer[512:])], [buffer[1:513]])):
        with pytest.raises(ValueError, match="overlap"):
            sp.adamw_plan(params, grads, [s, r][:len(params)])
    if bits == 32:
        with pytest.raises(ValueError, match="overlap"):
            sp.adamw_plan([a], [s.m], [s])
    sp.adamw_plan([a, b], [g, g], [s, r])  # (one gradient of two parameters is read twice)
    sp.adamw_plan([a], [a], [s])           # (each element is its own)
    sp.adamw_plan([host(buffer[:512])], [buffer[512:]], [s])
    sp.adamw_plan([host(buffer[:0]), a], [buffer[:0], g], [sp.adam_state(buffer[:0], bits), r])


def test_a_gradient_exchanged_for_a_parameter_is_refused():
    plan, params, grads = plan_of((8, 8), (64,))
    grads[0].data = params[1].data
    for _ in range(2):
        with pytest.raises(ValueError, match="overlap"):
            plan._follow()


def test_a_gradient_that_autograd_replaced_is_refused():
    # (a plan over p.grad: set to None and made anew, the plan's tensor is the old gradient)
    params = [host(torch.zeros(6)).requires_grad_() for _ in range(2)]
    for p in params:
        p.grad = torch.ones(6)
    plan = sp.adamw_plan(params, [p.grad for p in params], [sp.adam_state(p) for p in params])
    plan._follow()
    old = params[1].grad
    for new in (None, torch.ones(6)):
        params[1].grad = new
        with pytest.raises(ValueError, match="grad"):
            plan._follow()
    params[1].grad = old
    params[1].grad.data = torch.full((6,), 2.0)
    plan._follow()
    assert plan._calls[0][1][1].grad == old.data_ptr()
    # (tensors of its own: what autograd holds beside them is another's)
    other = sp.adamw_plan(params, [torch.ones(6) for _ in params], [sp.adam_state(p) for p in params])
    params[0].grad = None
    other._follow()


def test_a_step_counts_as_a_change_of_all_that_it_writes(monkeypatch):
    from paper_2608_09713_amd import training

    class Library:
        @staticmethod
        def spsyrk_adamw(*_):
            return 0

    monkeypatch.setattr(sp, "_lib", Library)
    monkeypatch.setattr(training, "_raw_stream", lambda device: 0)
    w = host(torch.ones(8, dtype=torch.bfloat16))
    master, g = torch.ones(8), torch.ones(8, dtype=torch.bfloat16)
    state = sp.adam_state(w)
    with torch.inference_mode():
        frozen = torch.ones(8)  # (has no count of its changes)
    plan = sp.adamw_plan([w, host(frozen)], [g, frozen.clone()], [state, sp.adam_state(frozen)], [master, None])
    x = torch.ones(8, requires_grad=True)
    saved = [(x * t).sum() for t in (w, master, state.m, state.v)]
    kept = (x * g).sum()
    w.requires_grad_()  # (after the plan was made)
    own = (w * w).sum()
    plan.step(1e-3, 1)
    for loss in (*saved, own):
        with pytest.raises(RuntimeError, match="inplace"):
            loss.backward()
    kept.backward()


def test_what_a_plan_refuses_when_it_is_made():
    p, s = host(torch.zeros(6, 6)), sp.adam_state(torch.zeros(6, 6))
    g = torch.ones(6, 6)
    with pytest.raises(ValueError, match="contiguous"):
        sp.adamw_plan([p], [g.t()], [s])
    with pytest.raises(ValueError, match="contiguous"):
        sp.adamw_plan([p], [g], [sp.AdamState(s.m, s.v.t())])
    with pytest.raises(ValueError, match="storage"):
        sp.adamw_plan([p], [torch.ones((6, 6), device="meta")], [s])
    empty = g.clone()
    empty.untyped_storage().resize_(0)
    with pytest.raises(ValueError, match="storage"):
        sp.adamw_plan([p], [empty], [s])
    with pytest.raises(TypeError):
        sp.adamw_plan([p], [None], [s])
    with pytest.raises(TypeError):
        sp.adamw_plan([p], [g.double()], [s])
    with pytest.raises(ValueError, match="size"):
        sp.adamw_plan([p], [g[:5]], [s])
    with pytest.raises(TypeError, match="master"):
        sp.adamw_plan([p], [g], [s], [g.clone()])
    plan = sp.adamw_plan([], [], [])
    assert plan._calls == [] and plan.step(1e-3, 1) is None
    # storage given back and taken again, as by programs that keep parameters elsewhere between steps
    plan = sp.adamw_plan([p], [g], [s])
    g.untyped_storage().resize_(0)
    with pytest.raises(ValueError, match="storage"):
        plan._follow()
    g.untyped_storage().resize_(36 * 4)
    plan._follow()
    assert plan._calls[0][1][0].grad == g.data_ptr()
