"""The next k-mer of a read.

Reads are rows of a k-mer matrix (CSR, one column per k-mer); a model of one
block learns which column follows another in a row.  A k-mer's vector is looked
up (``embed``), a block mixes it, its output is normed, gated and added to the
vector, and the sum normed again (``block_norm``); the loss over all columns and
its gradients come without the logits being kept (``linear_cross_entropy_grad``).
``block_norm_grad`` and ``embed_grad`` carry them back, and one ``adamw`` plan
steps all parameters.

    python examples/kmer_model.py
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_09713_amd as sp  # noqa: E402
from paper_2608_09713_amd import workloads  # noqa: E402

SCALE = 0.5  # of the block's output in the sum


def followers(A):
    """(tokens, targets): the pairs of consecutive columns of a DeviceCSR's rows."""
    cols = A.col_idx[:A.nnz].long()
    last = torch.zeros(A.nnz, dtype=torch.bool, device=cols.device)
    ends = A.row_ptr[1:][A.row_ptr[1:] > A.row_ptr[:-1]] - 1
    last[ends] = True
    return cols[:-1][~last[:-1]], cols[1:][~last[:-1]]


def parameters(columns, dim, device, seed=1, dtype=torch.float32):
    gen = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape, scale):
        return (torch.randn(shape, device=device, generator=gen) * scale).to(dtype)

    ones = torch.ones(dim, device=device, dtype=dtype)
    return dict(table=normal(columns, dim, scale=1.0), mix=normal(dim, dim, scale=dim ** -0.5), gate=ones.clone(),
                post=ones.clone(), pre=ones.clone(), out=normal(columns, dim, scale=dim ** -0.5))


def gradients(p, tokens, targets, weight=None):
    """(loss of every pair, {name: gradient} of ``(weight * loss).sum()``)."""
    x = sp.embed(tokens, p["table"])
    block = x @ p["mix"]
    y, h, r1, r2 = sp.block_norm(x, block, p["gate"], SCALE, p["post"], p["pre"])
    loss, dh, dout = sp.linear_cross_entropy_grad(h, p["out"], targets, row_weight=weight)
    dx, dblock, dgate, dpost, dpre = sp.block_norm_grad(None, dh, y, block, r1, r2, p["gate"], SCALE, p["post"], p["pre"])
    dtable = sp.embed_grad(tokens, dx + dblock @ p["mix"].t(), p["table"].shape[0])
    return loss, dict(table=dtable, mix=x.t() @ dblock, gate=dgate, post=dpost, pre=dpre, out=dout)


def train(rows=2048, columns=1 << 14, dim=128, steps=20, batch=4096, rate=1e-2, bits=32, device="cuda:0", log=print):
    """Losses of the steps (mean over the batch); bits: of the optimiser's states."""
    A = sp.DeviceCSR.from_host(workloads.kmer(rows, columns, 16, workloads.rng_for(7, 1, 0)), device)
    tokens, targets = followers(A)
    p = parameters(columns, dim, device)
    grads = {k: torch.empty_like(v) for k, v in p.items()}
    plan = sp.adamw_plan(p.values(), grads.values(), [sp.adam_state(v, bits) for v in p.values()])
    gen = torch.Generator(device=device).manual_seed(2)
    weight = torch.full((batch,), 1.0 / batch, device=device)
    losses = []
    for step in range(1, steps + 1):
        pick = torch.randint(0, tokens.numel(), (batch,), device=device, generator=gen)
        loss, new = gradients(p, tokens[pick], targets[pick], weight)
        for k, g in grads.items():
            g.copy_(new[k])
        plan.step(rate, step)
        losses.append(float(loss.mean()))
        if log:
            log(f"step {step}: loss {losses[-1]:.4f}", flush=True)
    return losses


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--rows", type=int, default=2048)
    a.add_argument("--columns", type=int, default=1 << 14)
    a.add_argument("--dim", type=int, default=128)
    a.add_argument("--steps", type=int, default=20)
    a.add_argument("--batch", type=int, default=4096)
    a.add_argument("--state-bits", type=int, default=32, choices=(8, 32))
    args = a.parse_args()
    train(args.rows, args.columns, args.dim, args.steps, args.batch, bits=args.state_bits)
