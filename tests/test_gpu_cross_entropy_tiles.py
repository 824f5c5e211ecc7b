"""The gradient's products of the cross entropy at sizes that take the largest tiles,
many steps of k, split products, and rows in several turns.

The plain 64-bit form (``training_reference``) runs on the GPU, some rows at a time;
tolerances are those of ``test_gpu_cross_entropy``.
"""
import pytest
import torch

import paper_2608_09713_amd as sp
from tests import training_reference as ref
from tests.test_gpu_cross_entropy import errors
from tests.test_gpu_rows import DEV, ROUND, TINY, U

pytestmark = pytest.mark.gpu
HALF = [torch.float16, torch.bfloat16]


@pytest.fixture(scope="module", autouse=True)
def _library():
    sp.library()
    yield
    torch.cuda.empty_cache()


def problem(N, V, D, dtype, seed=0):
    g = torch.Generator(device=DEV).manual_seed(1000 * seed + N + V + D)

    def rand(*shape):
        return torch.rand(shape, generator=g, device=DEV)

    w = (torch.randn((V, D), generator=g, device=DEV) * (2.0 / D ** 0.5)).to(dtype)
    t = torch.randint(0, V, (N,), generator=g, device=DEV)
    x = (torch.randn((N, D), generator=g, device=DEV) + w[t].float() * rand(N, 1) * 4.0).to(dtype)
    t[rand(N) < 0.2] = -1
    wt = rand(N) * 2 - 0.5
    wt[rand(N) < 0.2] = 0.0
    return x, w, t, wt


def reference(x, w, t, wt):
    """ref.cross_entropy, a part of the rows at a time."""
    rows = max(1, 1 << 27 >> w.shape[0].bit_length())
    over = ("dw", "dw_mag", "q_dw", "x_abs")
    parts, sums = [], {}
    w = w.double()
    for r in range(0, x.shape[0], rows):
        s = slice(r, r + rows)
        d = ref.cross_entropy(x[s].double(), w, t[s], 1.0, wt[s].double())
        for k in over:
            v = d.pop(k)
            sums[k] = sums[k].add_(v) if k in sums else v
        parts.append(d)
    one = {k: torch.cat([p[k] for p in parts]) for k in parts[0] if k != "w_abs"}
    return dict(one, w_abs=parts[0]["w_abs"], **sums)


def within(got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol)
    assert got.shape == want.shape and not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off"


def compare(got, want, wt, N, V, D, dtype):
    loss, dx, dw = got
    ez, e_lse, e_loss = errors(want, V, D)
    within(loss, want["loss"], torch.where(want["named"], e_loss, 0.0) + TINY[torch.float32], "loss")
    r = ROUND[dtype]
    rel = float(((ez + e_lse) * 2 + 10 * U + 4 * U * (want["lse"].abs() + want["zmag"])).max())
    lost = 2.0 ** -38 * float(wt.abs().max()) if dtype == torch.float16 else 0.0
    for name, out, terms, each in (("dx", dx, V, "w_abs"), ("dw", dw, N, "x_abs")):
        tol = ((r * 1.01 + rel + (terms + 4) * U) * want[name + "_mag"] + (r * 1.01 + rel) * want["q_" + name]
               + lost * want[each])
        within(out, want[name], tol + r * (want[name].abs() + tol) + TINY[dtype], name)
    assert not dx[~want["used"]].any()


def run(N, V, D, dtype):
    x, w, t, wt = problem(N, V, D, dtype)
    got = sp.linear_cross_entropy_grad(x, w, t, 1.0, wt)
    compare(got, reference(x, w, t, wt), wt, N, V, D, dtype)


# (16-bit products by 256 x 256: dW over 5 and 16 steps of k, dX split; dX whole over 16 and
# 17 steps; W, x and the outputs on boundaries in whole steps, and odd)
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("N,V,D", [(300, 12544, 1024), (1000, 12300, 1001), (1003, 12544, 1024), (6200, 1024, 2048),
                                   (6203, 1033, 2001)])
def test_largest_tiles_of_16_bits(dtype, N, V, D):
    run(N, V, D, dtype)


# (and in 32 bits beside them: 128 x 128 and 128 x 64 over many steps)
@pytest.mark.parametrize("N,V,D", [(1000, 12300, 1001), (6203, 1033, 2001)])
def test_many_steps_of_32_bits(N, V, D):
    run(N, V, D, torch.float32)


# (three turns of 2^17 rows: the first one's sums are added to by the second and rounded by the third)
@pytest.mark.parametrize("dtype", [torch.float32, *HALF])
def test_three_turns(dtype):
    N, V, D = 2 * (1 << 17) + 300, 331, 197
    run(N, V, D, dtype)


# (turns cut by their 2 GB: several rows of large tiles, with columns past their ends)
@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 300), (torch.float16, 320), (torch.float32, 45)])
def test_turns_of_many_columns(dtype, D):
    V = 1100003
    turn = (1 << 31) // dtype.itemsize // (V + 63) // 256 * 256
    run(2 * turn + 100, V, D, dtype)
