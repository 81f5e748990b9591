"""What the compiler made of the training kernels: the registers and LDS that their launches count on."""
import re

import pytest

from test_kernel_resources import kernels      # noqa: F401


def some(kernels, pattern):      # noqa: F811
    return {n: k for n, k in kernels.items() if re.search(pattern, n)}


@pytest.mark.parametrize("pattern", [r"norm_grad_kernel", r"norm_grad_router_kernel", r"norm_grad_sum_kernel", r"train_norm_kernel",
                                     r"router_rows_kernel", r"balance_(sums|grad|one)_kernel", r"combine_grad_kernel"])
def test_no_scratch(kernels, pattern):      # noqa: F811
    found = some(kernels, pattern)
    assert found
    for n, k in found.items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, n


def test_wavefronts_that_share_a_cu(kernels):      # noqa: F811
    """Of the gradient's kernels a CU has one workgroup of 16 or 8 wavefronts, or two of four; of the forward ones 16 wavefronts, 8 with the
    weights of many experts."""
    for n, k in some(kernels, r"norm_grad_kernel").items():
        threads = k[".max_flat_workgroup_size"]
        assert threads in (512, 1024) and k[".vgpr_count"] + k[".agpr_count"] <= (128 if threads == 1024 else 256), n
        assert k[".group_segment_fixed_size"] <= 160 * 1024, n
        if "ELi512E" in n:                                   # rows of several wavefronts: two workgroups of four
            assert k[".group_segment_fixed_size"] <= 80 * 1024, n
    for n, k in some(kernels, r"train_norm_kernel").items():
        many = re.search(r"ELi8ELb[01]E", n) is not None
        assert k[".vgpr_count"] + k[".agpr_count"] <= (256 if many else 160), n
        assert k[".group_segment_fixed_size"] <= 80 * 1024, n
    for n, k in some(kernels, r"combine_grad_kernel").items():
        assert k[".vgpr_count"] <= 64, n
