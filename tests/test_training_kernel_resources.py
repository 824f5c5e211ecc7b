"""Register budgets of a training step's kernels, read from the compiler's resource
report for gfx950 (no GPU needed).

The products of 256 x 256 tiles hold 128 sums and two half steps' fragments a lane
and have 256 registers (two wavefronts per SIMD): spills there would wait for the
loads that are under way.  Their two buffers leave room on a compute unit for one
workgroup.  Of the gradient of the norms around a block, which has 128 registers
where two workgroups of 512 threads are to share a compute unit, at most 48 bytes a
lane spill.  AdamW's kernels do not spill, and keep eight wavefronts a SIMD with
states of 32 bits.
"""
from tests.test_kernel_resources import _report, pytestmark  # noqa: F401


def test_cross_entropy_budgets():
    ks = _report("crossentropy.hip")
    products = {k: v for k, v in ks.items() if "logits_kernel" in k or "product_kernel" in k}
    assert len(products) == 3 * 2 * (2 + 4)
    for name, r in products.items():
        assert r["Occupancy"] >= 1 and r["LDS"] <= 160 * 1024, (name, r)
    for name, r in ks.items():
        assert r["ScratchSize"] == 0, (name, r)


def test_block_norm_budgets():
    ks = _report("blocknorm.hip")
    grads = {k: v for k, v in ks.items() if "after_block_grad" in k and "long" not in k}
    assert len(grads) > 50
    for name, r in ks.items():
        assert r["ScratchSize"] <= (48 if name in grads and "Li512E" in name else 0), (name, r)
        if name in grads and "Li0ELi512E" in name:
            assert r["Occupancy"] >= 4, (name, r)


def test_adamw_budgets():
    ks = _report("adamw.hip")
    assert len([k for k in ks if "adamw_wide" in k]) == len([k for k in ks if "adamw_narrow" in k]) == 9
    for name, r in ks.items():
        assert r["ScratchSize"] == 0 and r["Occupancy"] >= (8 if "adamw_wide" in name else 4), (name, r)


def test_products_keep_two_wavefronts_a_simd():
    # (by registers and by LDS: one workgroup of eight wavefronts or two of four on a compute unit)
    products = {k: v for k, v in _report("crossentropy.hip").items() if "logits_kernel" in k or "product_kernel" in k}
    for name, r in products.items():
        assert r["Occupancy"] >= 2 and r["VGPRs"] <= 256, (name, r)
        assert r["LDS"] * (1 if "Li8ELi4ELi2ELi4E" in name else 2) <= 160 * 1024, (name, r)
    assert sum("Li8ELi4ELi2ELi4E" in k for k in products) == 12
