"""The residual branch: equal to the separate operators, bit for bit, forward
and backward; in evaluation, frozen, without a bias."""

import pytest
import torch

from gpu_util import say
from paper_2609_02846_amd.dropout import dropout
from paper_2609_02846_amd.fp8 import fp8_linear
from paper_2609_02846_amd.norm import layer_norm
from paper_2609_02846_amd.operators import layer_norm_grad
from paper_2609_02846_amd.sublayer import PreNormSublayer, sublayer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale,grad", [("e8m0", "e4m3"), ("f32", "e5m2")])
@pytest.mark.parametrize("bias", [True, False])
def test_equals_the_separate_calls(scale, grad, bias):
    for T, C in [(1, 64), (40, 300), (260, 512)]:
        say("sublayer", scale, grad, bias, T, C)
        g = torch.Generator().manual_seed(T)
        rand = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()  # noqa: E731
        x, w, dout = rand(T, C).requires_grad_(), rand(C, C).requires_grad_(), rand(T, C)
        gain, b = rand(C).requires_grad_(), rand(C).requires_grad_() if bias else None
        leaves = [t for t in (x, gain, b, w) if t is not None]
        out = sublayer(x, gain, b, w, 0.2, 5, 6, 1e-5, scale, grad)
        got = torch.autograd.grad(out, leaves, dout)
        xs = x.detach().requires_grad_()
        h = layer_norm(xs, gain, b, 1e-5)
        hs = h.detach().requires_grad_()
        y = dropout(fp8_linear(hs, w, scale, grad), 0.2, 5, 6, residual=xs)
        assert torch.equal(out, y)
        dh, dw = torch.autograd.grad(y, (hs, w), dout)
        from paper_2609_02846_amd.operators import layer_norm_forward
        _, mean, rstd = layer_norm_forward(xs.detach(), gain.detach(), b, 1e-5, stats=True)
        dx, dg, db = layer_norm_grad(xs.detach(), dh, gain.detach(), mean, rstd, residual_grad=dout)
        want = [dx, dg] + ([db] if bias else []) + [dw]
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_module():
    m = PreNormSublayer(384, p=0.1, seed=3)
    x = torch.randn(2, 50, 384, device="cuda").to(torch.bfloat16).requires_grad_()
    a, b = m(x), m(x)
    assert a.shape == x.shape and not torch.equal(a, b)            # another key each call
    a.float().sum().backward()
    assert x.grad is not None and all(p.grad is not None for p in m.parameters())
    m.eval()
    with torch.no_grad():
        want = x + m.linear(m.norm(x))
        assert torch.equal(m(x), want)
        m.linear.freeze()
        assert torch.equal(m(x), want)
