"""Registers that the launches of LayerNorm of training count on: 16 wavefronts to a CU are four to a SIMD, of 128 registers each."""
import re

import pytest

from test_kernel_resources import kernels      # noqa: F401


def registers(kernels, pattern):      # noqa: F811
    found = {n: k[".vgpr_count"] + k[".agpr_count"] for n, k in kernels.items() if re.search(pattern, n)}
    assert found
    return found


def test_sixteen_wavefronts_to_a_cu_of_the_norm_but_where_its_launch_says_so(kernels):      # noqa: F811
    """Not of the weights of many experts, and of one shape, with a router of two and not all outputs, 12."""
    twelve = re.compile(r"train_norm_kernelIf(f|DF16_|DF16b)NS_8RowShapeILi4ELi4ELi(64|512)ELi3EEELi2ELb0E")
    for n, count in registers(kernels, r"train_norm_kernel.*ELi[02]ELb[01]E").items():
        assert count <= (168 if twelve.search(n) else 128), (n, count)


@pytest.mark.parametrize("pattern", [r"train_norm_kernel.*ELi8ELb[01]E", r"norm_grad_kernel.*RowShapeILi\dELi\dELi\d+ELi\dEEELi8E"])
def test_eight_wavefronts_to_a_cu_of_many_experts(kernels, pattern):      # noqa: F811
    for n, count in registers(kernels, pattern).items():
        assert count <= 256, (n, count)
