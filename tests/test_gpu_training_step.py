"""A training step's operators together, as a program runs them: one behind the
other, captured and replayed, on another stream, from two threads.

The step's gradients are compared with 64-bit autograd.  Tolerance, fixed from
the arithmetic: each of the five operators and three products between them has
an error of at most 512 u (u = 2^-24) of the magnitude of its terms, which what
cancels in it may exceed the result's by at most 32 (norms of 64 columns, sums
over 300 rows): 8 * 512 * 32 u = 2^-7 of the gradient's largest entry.
"""
import threading

import pytest
import torch

import examples.kmer_model as example
import paper_2608_09713_amd as sp
from tests.test_gpu_rows import DEV, gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    sp.library()


def problem(n=300, columns=500, dim=64, dtype=torch.float32):
    g = gen(n)
    tokens = torch.randint(0, columns, (n,), generator=g)
    targets = torch.randint(0, columns, (n,), generator=g)
    targets[::7] = -1
    weight = torch.rand(n, generator=g) / n
    p = {k: v.to(dtype) for k, v in example.parameters(columns, dim, "cpu").items()}
    return p, tokens, targets, weight


def test_gradients_of_a_step():
    p, tokens, targets, weight = problem()
    loss, grads = example.gradients({k: v.to(DEV) for k, v in p.items()}, tokens.to(DEV), targets.to(DEV), weight.to(DEV))
    q = {k: v.double().requires_grad_() for k, v in p.items()}
    x = q["table"][tokens]
    b = x @ q["mix"]
    u = b / torch.sqrt(b.square().mean(1, keepdim=True) + 1e-6) * q["post"]
    y = x + example.SCALE * q["gate"] * u
    h = y / torch.sqrt(y.square().mean(1, keepdim=True) + 1e-6) * q["pre"]
    z = h @ q["out"].t()
    want = torch.where(targets >= 0, torch.logsumexp(z, 1) - z.gather(1, targets.clamp(min=0)[:, None])[:, 0], 0.0)
    (weight.double() * want).sum().backward()
    assert (loss.cpu().double() - want).abs().max() <= 2.0 ** -7
    for k, v in q.items():
        assert (grads[k].cpu().double() - v.grad).abs().max() <= 2.0 ** -7 * v.grad.abs().max(), k


@pytest.mark.parametrize("bits", [32, 8])
def test_example_runs(bits):
    losses = example.train(rows=256, columns=1 << 10, dim=32, steps=3, batch=128, bits=bits, log=None)
    assert len(losses) == 3 and all(map(lambda v: v == v and abs(v) < 1e6, losses))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_two_captured_steps(dtype):
    # two graphs, each a whole step of its own parameters, replayed in turn with
    # eager steps between: every replay has the eager result
    sets = []
    for k in range(2):
        p, tokens, targets, weight = problem(200 + 31 * k, 300, 40, dtype)
        args = ({n: v.to(DEV) for n, v in p.items()}, tokens.to(DEV), targets.to(DEV), weight.to(DEV))
        states = [sp.adam_state(v, 8 if k else 32) for v in args[0].values()]
        sets.append((args, states))

    def step(args, states):
        loss, grads = example.gradients(*args)
        sp.adamw(list(args[0].values()), list(grads.values()), states, 1e-3, 5)
        return loss

    def copy(args, states):
        return (({n: v.clone() for n, v in args[0].items()}, *args[1:]),
                [sp.AdamState(*(None if t is None else t.clone() for t in s)) for s in states])

    eager = [copy(*s) for s in sets]
    stream, graphs, losses = torch.cuda.Stream(), [], []
    for s in sets:  # (the products' first calls set up their library outside of the graphs)
        step(*copy(*s))
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for s in sets:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                losses.append(step(*s))
            graphs.append(graph)
    torch.cuda.current_stream().wait_stream(stream)
    for turn in range(3):
        for graph, loss, s, e in zip(graphs, losses, sets, eager):
            graph.replay()
            want = step(*e)
            torch.cuda.synchronize()
            assert torch.equal(loss, want)
            for a, b in zip(s[0][0].values(), e[0][0].values()):
                assert torch.equal(a, b)
            for a, b in zip(s[1], e[1]):
                assert all(torch.equal(u, v) for u, v in zip(a, b) if u is not None)


def calls(seed):
    p, tokens, targets, weight = problem(257 + seed, 700, 72)
    p = {k: v.to(DEV) for k, v in p.items()}
    args = (p, tokens.to(DEV), targets.to(DEV), weight.to(DEV))
    return lambda: [v for v in example.gradients(*args)[1].values()]


def test_another_stream():
    run = calls(0)
    want = run()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = run()
    torch.cuda.current_stream().wait_stream(stream)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_two_threads():
    runs = [calls(k) for k in range(2)]
    want = [run() for run in runs]
    torch.cuda.synchronize()
    got, errors = [[], []], []

    def work(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(5):
                    got[k].append(runs[k]())
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # (told to the test's thread)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for k in range(2):
        for each in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(want[k], each))
