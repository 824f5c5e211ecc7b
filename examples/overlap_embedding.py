"""Vectors of reads that reproduce their overlaps.

Reads are rows of a k-mer matrix A (CSR, one column per k-mer).  The Jaccard
similarities of all pairs that share a k-mer come from ``lower`` and
``mirror``; their rows are the teacher.  The student has a vector per k-mer: a
read's vector is the sum of its k-mers' (``embed``), normalised
(``layer_norm``), and the logits of read i are the products of its vector with
those of all reads.  ``distill_grad`` gives the loss and the logits' gradient,
``layer_norm_grad`` and ``embed_grad`` carry it back to the k-mers' vectors.

    python examples/overlap_embedding.py
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_09713_amd as sp  # noqa: E402
from paper_2608_09713_amd import workloads  # noqa: E402


def train(rows=4096, columns=1 << 15, dim=128, steps=20, rate=0.5, temperature=0.25, device="cuda:0", log=print):
    """Losses of the steps (mean over the reads that overlap others)."""
    A = sp.DeviceCSR.from_host(workloads.kmer(rows, columns, 16, workloads.rng_for(7, 1, 0)), device)
    J = sp.mirror(sp.lower(A, "jaccard"), "jaccard")
    gen = torch.Generator(device=device).manual_seed(1)
    table = torch.randn((columns, dim), device=device, generator=gen) * 0.1
    gamma, beta = torch.ones(dim, device=device), torch.zeros(dim, device=device)
    scale = A.nrows / max(A.nnz, 1)  # (1 / a read's k-mers)
    overlaps = (J.row_ptr[1:] - J.row_ptr[:-1]) > 1
    weight = overlaps.float() / overlaps.sum().clamp(min=1)
    losses = []
    for step in range(steps):
        bags = sp.embed(A, table, scale)
        x, mean, rstd = sp.layer_norm(bags, gamma, beta)
        logits = x @ x.T / dim ** 0.5
        loss, dlogits = sp.distill_grad(logits, J, temperature, weight)
        dx = (dlogits @ x + dlogits.T @ x) / dim ** 0.5
        dbags, dgamma, dbeta = sp.layer_norm_grad(dx, bags, mean, rstd, gamma, beta)
        dtable = sp.embed_grad(A, dbags, columns, scale)
        table -= rate * dim * dtable
        gamma -= 0.1 * rate * dgamma
        beta -= 0.1 * rate * dbeta
        losses.append(float((weight * loss).sum()))
        if log:
            log(f"step {step}: loss {losses[-1]:.4f}", flush=True)
    return losses


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--rows", type=int, default=4096)
    p.add_argument("--columns", type=int, default=1 << 15)
    p.add_argument("--dim", type=int, default=128)
    p.add_argument("--steps", type=int, default=20)
    args = p.parse_args()
    train(args.rows, args.columns, args.dim, args.steps)
