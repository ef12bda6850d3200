"""Paged attention's weights add up to one: its values are divided by the sum of what the
product takes, P rounded to the inputs' type.  With values that are all 1 the output is 1."""

import pytest
import torch

from gpu_util import say
from paper_2609_02846_amd.attention import attention, paged_attention

pytestmark = pytest.mark.gpu


def pages_of(k, v, page):
    """Dense k and v [n, heads, dim] as a cache with one row's table and length."""
    n = k.shape[0]
    pages = -(-n // page)
    kc, vc = (torch.zeros(pages * page, *t.shape[1:], dtype=t.dtype, device="cuda") for t in (k, v))
    kc[:n], vc[:n] = k, v
    return (*(c.view(pages, page, *c.shape[1:]) for c in (kc, vc)), torch.arange(pages, dtype=torch.int32).cuda()[None],
            torch.tensor([n], dtype=torch.int32).cuda())


@pytest.mark.parametrize("dtype,low", [(torch.bfloat16, -0.0021), (torch.float16, -0.005287)])
@pytest.mark.parametrize("D", [64, 128])
def test_weights_that_are_all_rounded_down(dtype, low, D):
    """One key with P = 1 and 31 with P a little above 1/2, less than half a step of the
    type: 0.50178 (bf16, half a step 0.00195) and 0.50018 (fp16, 0.00024).  Divided by the
    sum before the rounding the output would be 16.5 / 16.555, or 16.5 / 16.5056, which
    is more than half a step below 1."""
    say("rounded down", dtype, D)
    q, k = (torch.zeros(n, 1, D, dtype=dtype, device="cuda") for n in (1, 32))
    q[..., :2] = 1.0
    k[1:, 0, 0], k[1:, 0, 1] = -0.6875, low
    v = torch.ones_like(k)
    p = torch.exp(k.double().sum(-1))[1:]
    half = torch.finfo(dtype).eps / 4                # (half a step of the numbers from 1/2 to 1)
    assert (p > 0.5 + 0.6 * half).all() and (p < 0.5 + 0.95 * half).all()
    o = paged_attention(q, *pages_of(k, v, 16), scale=1.0)
    assert torch.equal(o, torch.ones_like(o)), o.flatten()[:2].tolist()
    assert torch.equal(attention(q, k, v, scale=1.0), torch.ones_like(o))


@pytest.mark.parametrize("dtype,lens", [(torch.bfloat16, (1, 2, 5, 31, 33, 100, 129, 513, 1500, 5000)),
                                        (torch.float16, (1, 2, 5, 31, 33, 100, 129, 513, 1025, 1500))])
def test_values_of_one(dtype, lens):
    """Of any weights, through waves and parts: two sums of n numbers in binary32, each off by
    n 2^-24 at most, relative to half a step below 1 (2^-9 and 2^-12): 6e-4 of 1.9e-3, 1.8e-4
    of 2.4e-4."""
    for i, n in enumerate(lens):
        say("ones", dtype, n)
        g = torch.Generator().manual_seed(i)
        q, k = (torch.randn(m, 8 // h, 64, generator=g).to(dtype).cuda() for m, h in ((1, 1), (n, 4)))
        o = paged_attention(q, *pages_of(k, torch.ones_like(k), 16))
        assert torch.equal(o, torch.ones_like(o)), (n, (o.float() - 1).abs().max().item())
