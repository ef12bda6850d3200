"""The 8-bit layer where every quantity is exact: differences of the forward
pass have to equal the gradient."""

import pytest
import torch

from paper_2609_02846_amd.fp8 import fp8_linear

pytestmark = pytest.mark.gpu


def small(rows, cols, seed, top=2):
    """Whole numbers up to ``top``, with 4 in the first row and column: every
    block's largest is 4, and either kind of scale holds 0, 1, 2 and 4 exactly
    (E8M0: 64 times those; F32: 112 times in E4M3, 14336 times in E5M2)."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randint(-top, top + 1, (rows, cols), generator=g).float()
    x[0, :] = x[:, 0] = 4.0
    return x.to(torch.bfloat16).cuda()


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("grad", ["e4m3", "e5m2"])
def test_differences_are_the_gradient(scale, grad):
    """Y, dX and dW are sums of at most 15 products up to 16: whole numbers below
    256, which bf16 holds."""
    T, K, N = 14, 15, 12
    x, w = small(T, K, 1).requires_grad_(), small(N, K, 2).requires_grad_()
    dy = small(T, N, 3)
    dx, dw = torch.autograd.grad(fp8_linear(x, w, scale, grad), (x, w), dy)
    f = lambda a, b: (fp8_linear(a.detach(), b.detach(), scale, grad).double() * dy.double()).sum().item()  # noqa: E731
    for i, j in [(1, 1), (7, 14), (13, 8)]:
        for v, step, got in ((x, (i, j), dx), (w, (i % N, j), dw)):
            e = torch.zeros_like(v)
            e[step] = 1.0 if v[step] < 2 else -1.0   # stays within -2 .. 2
            sides = (f(x + e, w), f(x, w)) if v is x else (f(x, w + e), f(x, w))
            fd = (sides[0] - sides[1]) * e[step].item()
            assert abs(fd) < 256 and fd == got[step].item(), (step, fd, got[step].item())
    assert torch.equal(dx.float(), dy.float() @ w.detach().float())
    assert torch.equal(dw.float(), dy.float().t() @ x.detach().float())
