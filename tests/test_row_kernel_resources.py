"""Registers, scratch memory and LDS of the row kernels (layer norm, GELU, distillation): what their choice of workgroups is reckoned with."""
import re

from tests.test_kernel_resources import _wavefronts, kernels          # noqa: F401


def test_gradients_have_a_workgroup_of_1024_threads_on_a_compute_unit(kernels):       # noqa: F811
    """128 registers, no scratch memory (but for the widest rows of fp32) and at most a compute unit's LDS."""
    found = {name: use for name, uses in kernels.items() for use in uses if re.match(r"norm_grad_kernel<|gelu_kernel<\d, \d, true>", name)}
    assert len(found) == 22
    for name, use in found.items():
        assert use["threads"] == 1024 and use["vgpr"] <= 128 and use["lds"] <= 160 * 1024, (name, use)
        assert use["scratch"] <= (80 if name == "norm_grad_kernel<0, 1024, 16>" else 0), (name, use)


def test_gradients_of_short_batches_have_a_compute_unit_too(kernels):       # noqa: F811
    found = {name: use for name, uses in kernels.items() for use in uses if name.startswith("norm_short_grad_kernel<")}
    assert len(found) == 18
    for name, use in found.items():
        assert use["threads"] == 1024 and use["vgpr"] <= 128 and use["lds"] <= 160 * 1024, (name, use)
        assert use["scratch"] <= (32 if name == "norm_short_grad_kernel<0, 1024, 16>" else 0), (name, use)


def test_forward_row_kernels_use_no_scratch_memory(kernels):       # noqa: F811
    found = {name: use for name, uses in kernels.items() for use in uses if re.match(r"norm_(long_)?kernel<|norm_long_|gelu_kernel<\d, \d, false>|columns_kernel", name)}
    assert len(found) == 18 + 2 + 4 + 4 + 1
    for name, use in found.items():
        assert use["scratch"] == 0, (name, use)


def test_a_row_held_in_registers_is_held_there(kernels):       # noqa: F811
    found = {name: use for name, uses in kernels.items() for use in uses if name.startswith("distill_")}
    assert len(found) == 2 * 14 + 2 + 2 + 2 + 4
    for name, use in found.items():
        assert use["scratch"] == 0, (name, use)
    # four workgroups of the kernels that work on parts of rows on a compute unit: what rows are cut by
    for name in ("distill_slice_kernel<0, true>", "distill_slice_kernel<1, true>"):
        assert _wavefronts(found[name]) >= 4, found[name]
    for name in ("distill_part_kernel<0>", "distill_part_kernel<1>"):
        assert _wavefronts(found[name]) == 8, found[name]
    for name in ("distill_loss_kernel<0>", "distill_loss_kernel<1>"):
        assert _wavefronts(found[name]) >= 7, found[name]
