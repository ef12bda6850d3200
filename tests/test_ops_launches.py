"""The kernels that the 8-bit products and layer norm's backward pass launch,
and their workspaces, on the host alone (256 compute units)."""

import pytest

import test_gpu_fp8 as fp8_tests
from host_launches import fp8_call, launches, norm_grad_call, together


def names(calls):
    res = launches(calls)
    assert all(status == 0 for status, _ in res), res
    return [[next(n for n in KERNELS if n in k) for k, _, _ in kernels] for _, kernels in res]   # names may be mangled


KERNELS = ("quant_fp8_rows_kernel", "gemm_fp8_skinny_kernel", "gemm_fp8_wide_kernel", "gemm_fp8_kernel",
           "gemm_fp8_sum_kernel")
RING, SUM = "gemm_fp8_kernel", "gemm_fp8_sum_kernel"


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
def test_routes(scale):
    large = "gemm_fp8_wide_kernel" if scale == "e8m0" else RING
    for entry, first in (("gemm", []), ("linear", ["quant_fp8_rows_kernel"])):
        one, many = [["gemm_fp8_skinny_kernel"]], [first + ["gemm_fp8_skinny_kernel"]]
        call = lambda M, N, K: names([fp8_call(M, N, K, entry, scale=scale)])  # noqa: E731
        assert call(1, 21504, 4096) == one and call(8, 500, 1024) == one    # quantized where it is multiplied
        assert call(64, 21504, 4096) == many and call(17, 500, 1) == many and call(9, 500, 1024) == many
        assert call(65, 128, 1024) == [first + [RING]]
        assert call(100, 128, 2048) == [first + [RING, SUM]]                # few tiles, a long contraction
        assert call(8192, 21504, 4096) == [first + [large]]
    assert names([fp8_call(300, 300, 0, "linear", scale=scale)]) == [[RING]]


def test_tall_tiles_run_at_the_sizes_their_test_has():
    """The choice rests on modelled times: the test of the 256 x 128 tiles has to
    be at sizes that run on them, whole and split."""
    for M, N, K in fp8_tests.TALL:
        for scale, tiled in (("f32", False), ("f32", True), ("e8m0", False), ("e8m0", True)):
            (status, kernels), = launches([fp8_call(M, N, K, scale=scale, tiled=tiled)])
            assert status == 0 and kernels[0][2] == 512, (M, N, K, scale, kernels)      # eight waves
            assert ("sum" in kernels[-1][0]) == (K > 4096), (M, N, K, scale, kernels)


@pytest.mark.parametrize("call", [fp8_call(100, 128, 2048, capturing=True),
                                  fp8_call(100, 128, 2048, "linear", capturing=True),
                                  fp8_call(20, 128, 2048, "linear", capturing=True),
                                  norm_grad_call(4000, 500, capturing=True)])
def test_a_capture_without_a_workspace_enqueues_nothing(call):
    """Refused, with no launch recorded; after one eager call on the stream the
    capture holds the same launches."""
    eager = call[:-1] + "0"
    (s0, k0), (s1, k1), (s2, k2) = launches([call, eager, call])
    assert s0 != 0 and k0 == []
    assert s1 == s2 == 0 and k1 == k2 and len(k1) == len(launches([eager])[0][1]) > 1


def test_a_serving_call_grown_under_capture_enqueues_nothing():
    """The stream holds the workspace of a serving call of the same tokens whose
    product is not split, too small for the partial sums of this one."""
    grown = fp8_call(100, 128, 4096, "linear", capturing=True)
    (s0, k0), (s1, k1) = launches([fp8_call(100, 25600, 4096, "linear"), grown])
    assert s0 == 0 and len(k0) == 2 and s1 != 0 and k1 == []


@pytest.mark.parametrize("call,n", [(fp8_call(100, 128, 2048), 2), (fp8_call(100, 128, 2048, "linear"), 3),
                                    (fp8_call(20, 128, 2048, "linear"), 2), (norm_grad_call(4000, 500), 2)])
def test_launches_that_share_a_workspace_stay_together(call, n):
    status, kernels = launches([call])[0]
    assert status == 0 and len(kernels) == n, kernels
    assert together(4, 6, call) == (0, 24, 0)
