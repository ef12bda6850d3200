"""The test of the products' distance from their definition is at sizes that
run on every kernel (on the host alone, 256 compute units)."""

from host_launches import fp8_call, launches
from test_gpu_fp8_definition import ORDINARY


def test_every_kernel_is_among_them():
    for scale in ("f32", "e8m0"):
        seen = []
        for M, N, K, fused in ORDINARY:
            (status, kernels), = launches([fp8_call(M, N, K, "linear" if fused else "gemm", "f32", scale)])
            assert status == 0 and (not fused or len(kernels) == 1)
            name, _, threads = kernels[0]
            seen.append((name.split("gemm_fp8_")[1].split("kernel")[0], threads, len(kernels)))
        assert [s for s in seen if s[0] == "skinny_"] and (("", 256, 1) in seen) and (("", 256, 2) in seen) and \
            (("", 512, 1) in seen) and (("wide_", 256, 1) in seen) == (scale == "e8m0"), seen
