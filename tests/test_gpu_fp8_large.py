"""8-bit products and quantizers at sizes whose offsets pass 32 bits."""

import pytest
import torch

import paper_2609_02846_amd as ue
from gpu_util import say
from paper_2609_02846_amd.operators import scale_pitch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
def test_operand_past_32_bits(scale):
    """A payload of more than 4 GiB and a source of more than 2^32 elements'
    half: rows on both sides equal the same rows multiplied alone."""
    M, K, N = 2 ** 32 // 4096 + 300, 4096, 72
    say("fp8 large", M, K, N, scale)
    x = torch.randint(-64, 64, (M, K), dtype=torch.int8, device="cuda").to(torch.bfloat16)
    w = torch.randn(N, K, device="cuda").to(torch.bfloat16)
    p, s = ue.quantize_fp8(x, 1, "e4m3", scale)
    wp, ws, _, _ = ue.quantize_fp8_tiles(w, scale, transposed=False)
    y = ue.gemm_fp8("nt", M, N, K, p, s, wp, ws, out_dtype=torch.float32)
    edge = 2 ** 32 // K
    for r0 in (0, edge // 2 - 100, edge - 128, M - 200):
        sub = x[r0:r0 + 200].contiguous()
        p1, s1 = ue.quantize_fp8(sub, 1, "e4m3", scale)
        assert torch.equal(p1.view(torch.uint8), p[r0:r0 + 200].view(torch.uint8))
        assert torch.equal(s1[:, :200], s[:, r0:r0 + 200])
        want = ue.gemm_fp8("nt", 200, N, K, p1, s1, wp, ws, out_dtype=torch.float32)
        torch.testing.assert_close(y[r0:r0 + 200], want, rtol=1e-5, atol=1e-5 * want.abs().max().item())
    assert s.shape[1] == scale_pitch(M)


def test_output_past_32_bits():
    """C of more than 2^32 bytes, and a B operand of many rows."""
    M, N, K = 1100, 2 ** 20 + 77, 130
    say("fp8 large output", M, N, K)
    x = torch.randint(-8, 8, (M, K), dtype=torch.int8, device="cuda").to(torch.bfloat16)
    w = torch.randint(-8, 8, (N, K), dtype=torch.int8, device="cuda").to(torch.bfloat16)
    (p, s), (wp, ws, _, _) = ue.quantize_fp8(x, 1), ue.quantize_fp8_tiles(w, transposed=False)
    y = ue.gemm_fp8("nt", M, N, K, p, s, wp, ws, out_dtype=torch.float32)
    for m0, n0 in [(0, 0), (M - 40, N - 100), (M // 2, 2 ** 19), (M - 1, 5)]:
        want = x[m0:m0 + 40].float() @ w[n0:n0 + 100].float().t()       # whole numbers: exact
        assert torch.equal(y[m0:m0 + 40, n0:n0 + 100], want)
