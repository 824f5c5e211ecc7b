"""The AdamW step on the GPU against a plain 64-bit form.

Tolerances, fixed from the arithmetic: with u = 2^-24, m and v are sums of two
terms of positive weights, off by 4 u of the terms' magnitudes (rates, products,
sum; the scale of the gradient one more); the update is off by 8 u of itself and
what the errors of m and v (half of its own, under the root) pass on, and w by u
more of each term; 16-bit parameters by one rounding.  8-bit codes and scales are
those of the formula.
"""
import pytest
import torch

import paper_2608_09713_amd as sp
from tests import training_reference as ref
from tests.test_gpu_rows import DEV, DTYPES, ROUND, TINY, U, check, gen

pytestmark = pytest.mark.gpu
SIZES = [1, 7, 255, 256, 257, 0, 2048, 2049, 5000, 33, 12345]
LR, STEP, BETAS, EPS, DECAY = 3e-3, 7, (0.9, 0.99), 1e-8, 0.05


@pytest.fixture(scope="module", autouse=True)
def _library():
    sp.library()


def tensors(dtype, gdtype, bits, master, sizes, seed=3, shift=0):
    """Tensors one behind the other in one buffer each (so at any element's address)."""
    g = gen(seed)
    n = sum(sizes)

    def flat(t):
        buf = torch.zeros(n + shift, dtype=t.dtype, device=DEV)
        buf[shift:] = t.to(DEV)
        return list(torch.split(buf[shift:], sizes))

    w = torch.randn(n, generator=g) * 0.1
    p = w.to(dtype)
    grad = (torch.randn(n, generator=g) * torch.exp(torch.randn(n, generator=g) * 2) * 1e-2).to(gdtype)
    out = dict(p=p, g=grad, w=w if master else p.float())
    if bits == 32:
        m, v = torch.randn(n, generator=g) * 1e-2, torch.rand(n, generator=g) * 1e-3
        states = [sp.AdamState(a, b) for a, b in zip(flat(m), flat(v))]
        out.update(m=m, v=v)
    else:
        blocks = [-(-s // 256) for s in sizes]
        mc = torch.randint(-127, 128, (n,), generator=g).to(torch.int8)
        vc = torch.randint(0, 256, (n,), generator=g).to(torch.uint8)
        ms, vs = torch.rand(sum(blocks), generator=g) * 1e-2, torch.rand(sum(blocks), generator=g) * 1e-3
        scales = [list(torch.split(t.to(DEV), blocks)) for t in (ms, vs)]
        states = [sp.AdamState(*s) for s in zip(flat(mc), flat(vc), *scales)]
        parts = [ref.adam_decode(a, b, c, d) for a, b, c, d in
                 zip(torch.split(mc, sizes), torch.split(vc, sizes), torch.split(ms, blocks), torch.split(vs, blocks))]
        out.update(m=torch.cat([a for a, _ in parts]), v=torch.cat([b for _, b in parts]))
    return out, flat(p), flat(grad), states, flat(w) if master else None


def expect(out, scale=1.0, lr=LR, step=STEP):
    w, m, v = ref.adamw(out["w"].double(), out["g"].double() * scale, out["m"].double(), out["v"].double(), lr, step,
                        BETAS, EPS, DECAY)
    g = (out["g"].double() * scale).abs()
    em = 5 * U * (BETAS[0] * out["m"].double().abs() + (1 - BETAS[0]) * g) + 2.0 ** -149
    ev = 6 * U * v + 2.0 ** -149
    c1, c2 = 1 - BETAS[0] ** step, 1 - BETAS[1] ** step
    root = (v / c2).sqrt() + EPS
    update = (m / c1) / root
    e = lr * (em / c1 / root + (8 * U + ev / (v + 1e-300)) * update.abs()) + 3 * U * (out["w"].double().abs() + lr * update.abs())
    return (w, e), (m, em), (v, ev)


@pytest.mark.parametrize("dtype,gdtype,master", [(torch.float32, torch.float32, False)] + [
    (d, g, master) for d in DTYPES[1:] for g in (d, torch.float32) for master in (False, True)])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 3])
def test_step(dtype, gdtype, master, bits, shift):
    out, p, g, states, masters = tensors(dtype, gdtype, bits, master, SIZES, shift=shift)
    scale = torch.tensor([0.5], device=DEV) if shift else None
    sp.adamw(p, g, states, LR, STEP, BETAS, EPS, DECAY, scale, masters)
    (w, ew), (m, em), (v, ev) = expect(out, 0.5 if shift else 1.0)
    new = torch.cat(p).cpu()
    check(new, w, ew + ROUND[dtype] * (w.abs() + ew) + TINY[dtype], "param")
    if master:
        check(torch.cat(masters), w, ew, "master")
        assert torch.equal(new, torch.cat(masters).cpu().to(dtype))
    if bits == 32:
        check(torch.cat([s.m for s in states]), m, em, "m")
        check(torch.cat([s.v for s in states]), v, ev, "v")
        return
    values = sp.adam_values(states)
    at = 0
    for k, n in enumerate(SIZES):
        mc, vc, ms, vs = ref.adam_encode(m[at:at + n], v[at:at + n])
        at += n
        s = states[k]
        assert torch.equal(s.m_scale.cpu(), ms) and torch.equal(s.v_scale.cpu(), vs), n
        assert torch.equal(s.m.cpu(), mc) and torch.equal(s.v.cpu(), vc), n
        dm, dv = ref.adam_decode(mc, vc, ms, vs)
        check(values[k][0], dm, U * dm.abs() + 2.0 ** -149, "values of m")
        check(values[k][1], dv, U * dv.abs() + 2.0 ** -149, "values of v")


def test_more_tensors_than_a_launch_takes():
    sizes = [(k * 37) % 700 + 1 for k in range(130)]
    for bits in (32, 8):
        out, p, g, states, _ = tensors(torch.float32, torch.float32, bits, False, sizes)
        sp.adamw(p, g, states, LR, STEP, BETAS, EPS, DECAY)
        (w, ew), (m, _), (v, _) = expect(out)
        check(torch.cat(p), w, ew, "param")
        if bits == 8:
            at = 0
            for s, n in zip(states, sizes):
                mc, vc, _, _ = ref.adam_encode(m[at:at + n], v[at:at + n])
                assert torch.equal(s.m.cpu(), mc) and torch.equal(s.v.cpu(), vc)
                at += n


def test_kinds_of_tensors_together():
    a = tensors(torch.float32, torch.float32, 32, False, [100, 7])
    b = tensors(torch.bfloat16, torch.bfloat16, 8, False, [300])
    c = tensors(torch.float16, torch.float32, 32, False, [64])
    alone = []
    for out, p, g, s, _ in (a, b, c):
        q = [t.clone() for t in p]
        sp.adamw(q, g, [sp.AdamState(*(None if t is None else t.clone() for t in st)) for st in s], LR, STEP, BETAS, EPS, DECAY)
        alone += q
    sp.adamw([t for x in (a, b, c) for t in x[1]], [t for x in (a, b, c) for t in x[2]], [t for x in (a, b, c) for t in x[3]],
             LR, STEP, BETAS, EPS, DECAY)
    assert all(torch.equal(p, q) for p, q in zip([t for x in (a, b, c) for t in x[1]], alone))


def test_states_from_zero_and_many_steps():
    # 8 bits beside 32 from zero states: the first step's update is the gradient's sign
    n = 1000
    g = gen(9)
    w = torch.randn(n, generator=g).to(DEV)
    grads = [torch.randn(n, generator=g).to(DEV) for _ in range(5)]
    for bits in (32, 8):
        p, s = w.clone(), sp.adam_state(w, bits)
        sp.adamw([p], [grads[0]], [s], 1e-2, 1, weight_decay=0.0)
        assert ((w - p) / 1e-2 - grads[0].sign()).abs().max() < 1e-4
        for k in range(1, 5):
            sp.adamw([p], [grads[k]], [s], 1e-2, k + 1, weight_decay=0.0)
        assert torch.isfinite(p).all()
        if bits == 8:
            assert (s.v[grads[0] != 0] > 0).all()


def test_zero_and_tiny_and_broken_blocks():
    n = 256 * 5 + 10
    w = torch.ones(n, device=DEV)
    g = torch.zeros(n, device=DEV)
    g[256:512] = 1e-18       # (squares of 1e-36 (1 - beta2): a scale below the normal reciprocals' range)
    g[600] = float("inf")
    g[900] = float("nan")
    g[1024] = 1.0
    g[1025:1280] = 1e-9      # (far below the block's scale: codes of 0 for m, 1 for v)
    s = sp.adam_state(w, 8)
    p = w.clone()
    sp.adamw([p], [g], [s], 1e-2, 1, (0.9, 0.999), 1e-8, 0.0)
    m, v = sp.adam_values([s])[0]
    assert torch.equal(p[:256], w[:256]) and not s.m[:256].any() and not s.v[:256].any()
    assert (s.m[256:512] == 127).all() and (s.v[256:512] == 255).all()
    assert (m[256:512] - 1e-19).abs().max() < 1e-25
    assert torch.isnan(m[512:1024]).all() and torch.isnan(v[512:1024]).all()
    assert torch.isfinite(p[:512]).all() and torch.isfinite(p[1024:]).all() and torch.isnan(p[900])
    assert (s.m[1025:1280] == 0).all() and (s.v[1025:1280] == 1).all() and s.v[1024] == 255
    assert not s.m[1280:].any() and torch.equal(p[1280:], w[1280:])


def test_plan_follows_exchanged_storage_and_replays():
    out, p, g, states, _ = tensors(torch.bfloat16, torch.bfloat16, 32, False, [500, 77])
    plan = sp.adamw_plan(p, g, states)
    copies = [t.clone() for t in p], [sp.AdamState(s.m.clone(), s.v.clone()) for s in states]
    plan.step(LR, STEP, BETAS, EPS, DECAY)
    sp.adamw(copies[0], g, copies[1], LR, STEP, BETAS, EPS, DECAY)
    assert all(torch.equal(a, b) for a, b in zip(p, copies[0]))
    g[0].data = torch.randn(500, device=DEV).to(torch.bfloat16)
    plan.step(LR, STEP + 1, BETAS, EPS, DECAY)
    sp.adamw(copies[0], g, copies[1], LR, STEP + 1, BETAS, EPS, DECAY)
    assert all(torch.equal(a, b) for a, b in zip(p, copies[0]))
    # captured: the replays step as eager calls do
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            plan.step(LR, 9, BETAS, EPS, DECAY)
    torch.cuda.current_stream().wait_stream(stream)
    for _ in range(3):
        graph.replay()
        sp.adamw(copies[0], g, copies[1], LR, 9, BETAS, EPS, DECAY)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(p, copies[0]))


def test_overlapping_tensors_are_refused():
    w = torch.zeros(100, device=DEV)
    g, s, r = torch.zeros(100, device=DEV), sp.adam_state(w), sp.adam_state(w)
    with pytest.raises(ValueError, match="overlap"):
        sp.adamw([w, w], [g, g], [s, r], LR, 1)
    with pytest.raises(ValueError, match="overlap"):
        sp.adamw([w], [g], [sp.AdamState(s.m, s.m)], LR, 1)
    with pytest.raises(ValueError, match="overlap"):
        sp.adamw([w[:60], w[50:]], [g[:60], g[50:]], [sp.adam_state(w[:60]), sp.adam_state(w[50:])], LR, 1)


def test_exchanged_storage_of_another_size_or_type_is_refused():
    w, g = torch.zeros(100, device=DEV), torch.ones(100, device=DEV)
    plan = sp.adamw_plan([w], [g], [sp.adam_state(w)])
    before = g.data
    for other in (torch.ones(60, device=DEV), torch.ones(100, device=DEV, dtype=torch.bfloat16),
                  torch.ones(200, device=DEV)[::2]):
        g.data = other
        for _ in range(2):
            with pytest.raises((ValueError, TypeError)):
                plan.step(LR, 1)
    g.data = before
    plan.step(LR, 1, eps=0.0, weight_decay=0.0)
    assert (w + LR).abs().max() <= 2 ** -20 * LR  # (one step from zero: -lr)


def test_autograd_sees_the_change():
    w = torch.ones(8, device=DEV, requires_grad=True)
    loss = (w * w).sum()
    plan = sp.adamw_plan([w], [torch.ones(8, device=DEV)], [sp.adam_state(w)])
    plan.step(LR, 1)
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()
