"""AdamW over lists of tensors that differ in kind: with copies of some parameters.
Each tensor has the same bits as when it is stepped alone."""
import pytest
import torch

import paper_2608_09713_amd as sp
from tests.test_gpu_adamw import BETAS, DECAY, EPS, LR, STEP
from tests.test_gpu_rows import DEV, gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    sp.library()


def problem(kinds, bits, seed=4):
    """Parameters, gradients, states and copies of (size, type, with a copy)."""
    g = gen(seed)
    params = [torch.randn(n, generator=g).to(DEV).to(t) for n, t, _ in kinds]
    grads = [torch.randn(n, generator=g).to(DEV).to(t) for n, t, _ in kinds]
    masters = [p.float() if copy else None for p, (_, _, copy) in zip(params, kinds)]
    return params, grads, [sp.adam_state(p, bits) for p in params], masters


def same_as_alone(kinds, bits):
    params, grads, states, masters = problem(kinds, bits)
    for k in (1, 2):
        sp.adamw(params, grads, states, LR, k, BETAS, EPS, DECAY, masters=masters)
    q, g, s, w = problem(kinds, bits)
    for k in (1, 2):
        for i in range(len(kinds)):
            sp.adamw([q[i]], [g[i]], [s[i]], LR, k, BETAS, EPS, DECAY, masters=None if w[i] is None else [w[i]])
    for i, (n, _, copy) in enumerate(kinds):
        assert torch.equal(params[i], q[i]) and (not n or not torch.equal(params[i], problem(kinds, bits)[0][i]))
        assert all(a is b is None or torch.equal(a, b) for a, b in zip(states[i], s[i]))
        assert not copy or torch.equal(masters[i], w[i])


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("order", [1, -1])
def test_copies_of_some_parameters(bits, order):
    kinds = [(300, torch.bfloat16, True), (77, torch.float32, False), (4100, torch.float16, True), (9, torch.bfloat16, False)]
    same_as_alone(kinds[::order], bits)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("copy", [False, True])
def test_an_empty_tensor_in_front(bits, copy):
    same_as_alone([(0, torch.bfloat16, copy), (500, torch.bfloat16, copy), (0, torch.bfloat16, copy), (33, torch.bfloat16, copy)],
                  bits)


def test_a_change_at_the_same_address_is_refused_before_anything_is_stepped():
    w, g = torch.ones((64, 64), device=DEV), torch.ones((64, 64), device=DEV)
    state = sp.adam_state(w)
    plan = sp.adamw_plan([w], [g], [state])
    whole = w.data
    for other in (whole[:32], whole.t(), whole.view(torch.int32)):
        w.data = other
        for _ in range(2):
            with pytest.raises((ValueError, TypeError)):
                plan.step(LR, 1)
    assert (whole == 1).all() and not state.m.any()
    w.data = whole
    plan.step(LR, 1, weight_decay=0.0)
    assert (1 - whole - LR).abs().max() <= 2.0 ** -23  # (a first step of one rate, and a rounding near 1)
