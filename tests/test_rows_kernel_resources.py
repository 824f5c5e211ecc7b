"""Register budgets of the kernels between sparse rows and dense rows, read from
the compiler's resource report for gfx950 (no GPU needed).

The distillation kernel that holds a row in registers takes up to sixteen packs
a thread in workgroups of up to 1024 threads, which leaves 128 registers: none
of it spills.  The loss alone keeps two such workgroups on a compute unit (64
registers; 12 bytes a lane spill for 16-bit logits, which measures faster than
one workgroup).  The layer norm holds its rows without spills; its gradient
spills a little only for rows of more than 512 threads.  The sums of the lookup
keep four wavefronts per SIMD.
"""
import pytest

from tests.test_kernel_resources import _report, pytestmark  # noqa: F401


def test_distillation_budgets():
    ks = _report("distill.hip")
    fused = {k: v for k, v in ks.items() if "distill_fused" in k}
    rows = {k: v for k, v in ks.items() if "distill_rows" in k}
    assert len(fused) == 30 and len(rows) == 9
    for name, r in fused.items():
        assert r["ScratchSize"] == 0 and r["VGPRs"] <= 128, (name, r)
    for name, r in rows.items():
        two = "ELi1024EE" in name
        assert r["ScratchSize"] <= (12 if two else 0) and r["Occupancy"] >= (8 if two else 5), (name, r)


def test_layer_norm_budgets():
    ks = _report("norm.hip")
    norm = {k: v for k, v in ks.items() if "norm_kernel" in k}
    grad = {k: v for k, v in ks.items() if "norm_grad_kernel" in k}
    assert len(norm) == 55 and len(grad) > 40
    for name, r in norm.items():
        assert r["ScratchSize"] == 0 and r["Occupancy"] >= 5, (name, r)
    for name, r in grad.items():
        assert r["ScratchSize"] == 0 or "ELi1024E" in name, (name, r)


def test_lookup_budgets():
    ks = _report("embed.hip")
    sums = {k: v for k, v in ks.items() if "sums_kernel" in k}
    assert len(sums) == 12
    for name, r in ks.items():
        assert r["ScratchSize"] == 0, (name, r)
    for name, r in sums.items():
        assert r["Occupancy"] >= 4, (name, r)
    sort = [v for k, v in ks.items() if "sort_groups" in k]
    assert len(sort) == 1 and 2 * sort[0]["LDS"] <= 160 * 1024
