"""dS as two numbers in dK's product: pinned where the rest of the arithmetic is exact.

With keys of zeros and no mask every weight is 1 / n.  Output gradients come in threes that
add up to nothing, a, b and -(a + b), and with them each key's dS over the queries; with
queries that are all alike dK = scale q sum(dS) is 0, and what the kernel gives instead is
the error of delta = do . o and of dS."""

import pytest
import torch

import attention_model as model
from test_attention_rest import o_bounds

F, U = model.F, model.U[torch.bfloat16]
CASES = [(3, 3), (9, 40), (9, 300), (39, 39), (300, 130), (2049, 300), (30, 3000)]


def inputs(L, S, H, Hk, D, seed=0):
    g = torch.Generator().manual_seed(seed)
    eighths = lambda n, h, most: torch.randint(-most, most + 1, (n, h, D), generator=g) / 8  # noqa: E731
    q = torch.randn(1, H, D, generator=g).to(torch.bfloat16).expand(L, H, D).contiguous()
    a, b = eighths(L // 3, H, 7), eighths(L // 3, H, 7)
    do = torch.stack([a, b, -(a + b)], 1).reshape(L, H, D).to(torch.bfloat16)
    return q, torch.zeros(S, Hk, D, dtype=torch.bfloat16), (eighths(S, Hk, 15) + 0.5).to(torch.bfloat16), do


def exact(v, do):
    """(o, t, delta) in 64 bits, heads first; t = do . v."""
    v = v.double().transpose(0, 1).repeat_interleave(do.shape[1] // v.shape[1], 0)
    do = do.double().transpose(0, 1)
    o = (v.sum(1, keepdim=True) / v.shape[1]).expand(do.shape)
    return o, do @ v.transpose(1, 2), (do * o).sum(-1, keepdim=True)


def dk_bound(do, q, o, t, delta, Hk, scale):
    """How far dK may be from 0.  delta: that of o + o_rest, and a sum of D terms; dS: its
    difference and its product with P (off by less than 2^-17, which all rows and keys share),
    two numbers that leave U^2 of it, and the sums of two products over the rows of the
    heads that share the key; dK's own rounding."""
    L, H, D = do.shape
    n, group = t.shape[-1], H // Hk
    do = do.double().transpose(0, 1).abs()
    err = (do * o_bounds(o)[1]).sum(-1, keepdim=True) + (D + 2) * F * (do * o.abs()).sum(-1, keepdim=True)
    ds = (1 + 2.0 ** -17) / n * (err + (U * U * (1 + U) + (2 * L * group + 18) * F) * (t - delta).abs())
    bound = scale * (1 + 2 * U) * ds.sum(1)[:, :, None] * q[0].double().abs()[:, None]      # [H, n, D]
    return bound.view(Hk, group, n, D).sum(1).transpose(0, 1) + 1e-30


def heads_sum(x, Hk):
    return x.view(Hk, -1, *x.shape[1:]).sum(1)


@pytest.mark.parametrize("L,S", [(3, 3), (9, 40), (9, 300), (39, 39)])
def test_the_bound_sees_what_is_left_out(L, S):
    """dK with dS in one number, or from o as it was rounded, would be beyond the bound."""
    H, Hk, D = 4, 2, 16
    q, _, v, do = inputs(L, S, H, Hk, D)
    o, t, delta = exact(v, do)
    bound = dk_bound(do, q, o, t, delta, Hk, 0.25)
    rounded = lambda x: x.to(torch.bfloat16).double()  # noqa: E731
    two = lambda s: rounded(s) + rounded(s - rounded(s))  # noqa: E731
    dod, qd = do.double().transpose(0, 1), q.double().transpose(0, 1)

    def ratio(o, split):
        ds = split((t - (dod * o).sum(-1, keepdim=True)) / S)
        return (heads_sum(0.25 * ds.transpose(1, 2) @ qd, Hk).transpose(0, 1).abs() / bound).max().item()
    assert ratio(rounded(o) + rounded(o - rounded(o)), two) <= 1.0
    assert ratio(rounded(o) + rounded(o - rounded(o)), rounded) > 1.5


@pytest.mark.gpu
@pytest.mark.parametrize("L,S", CASES)
@pytest.mark.parametrize("D", [16, 64, 80, 128])
def test_on_the_gpu(L, S, D):
    from gpu_util import say
    from paper_2609_02846_amd.attention import attention

    say("dK's rest", L, S, D)
    H, Hk = 4, 2
    q, k, v, do = (t.cuda() for t in inputs(L, S, H, Hk, D, seed=D))
    o, t, delta = exact(v, do)
    leaves = [x.detach().requires_grad_() for x in (q, k, v)]
    dk, = torch.autograd.grad(attention(*leaves, causal=False), leaves[1:2], do)
    model.within(dk, torch.zeros_like(dk, dtype=torch.float64), dk_bound(do, q, o, t, delta, Hk, D ** -0.5), "dk")
