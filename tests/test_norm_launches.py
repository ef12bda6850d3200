"""Layer norm's launches at the sizes that its entry points take, on the host
alone."""

import pytest

from host_launches import launches, norm_grad_call


@pytest.mark.parametrize("cols", [2 ** 28 - 1, 2 ** 28, 2 ** 28 + 100, 2 ** 31 - 1])
def test_column_sums_of_the_widest_rows(cols):
    """A launch takes fewer than 2^32 work-items in one dimension."""
    (status, kernels), = launches([norm_grad_call(1, cols)])
    assert status == 0 and len(kernels) >= 3, kernels
    sums = [grid * 64 for name, grid, _ in kernels if "norm_sum_kernel" in name]
    assert cols <= sum(sums) < cols + 64 and len(sums) == len(kernels) - 2
