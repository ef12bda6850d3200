"""Gradients of attention under a window whose sinks many rows see from far away: rows
past the window in parts of their own, in long and short sequences, packed and of one
length, with more keys than queries and fewer."""

import pytest
import torch

import attention_model as model
from gpu_util import say
from paper_2609_02846_amd.attention import attention

pytestmark = pytest.mark.gpu


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()


def starts(lens, at=0):
    return (at + torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist())).to(torch.int32).cuda()


def check(q_lens, k_lens, Hq, Hk, D, window, sinks, batch=False, outside=0):
    say("sinks", q_lens, k_lens, Hq, Hk, D, window, sinks, batch, outside)
    T, S = sum(q_lens) + 2 * outside, sum(k_lens) + 2 * outside
    q, k, v = rand(1, T, Hq, D), rand(2, S, Hk, D), rand(3, S, Hk, D)
    do, mask = rand(4, T, Hq, D), dict(window=window, sinks=sinks)
    leaves = [t.requires_grad_() for t in (q, k, v)]
    if batch:
        n = len(q_lens)
        o = attention(*(t.view(n, -1, *t.shape[1:]) for t in leaves), **mask).view(q.shape)
    else:
        o = attention(*leaves, starts(q_lens, outside), starts(k_lens, outside), **mask)
    grads = torch.autograd.grad(o, leaves, do, retain_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(grads, torch.autograd.grad(o, leaves, do)))
    a = b = outside
    for L, M in zip(q_lens, k_lens):
        rows, keys = slice(a, a + L), slice(b, b + M)
        want = model.Sequence(q[rows].detach(), k[keys].detach(), v[keys].detach(), D ** -0.5, **mask)
        w, bound = want.gradients(do[rows])
        model.within(grads[0][rows], w[0], bound[0], f"{L} x {M} dq")
        model.within(grads[1][keys], w[1], bound[1], f"{L} x {M} dk")
        model.within(grads[2][keys], w[2], bound[2], f"{L} x {M} dv")
        a, b = a + L, b + M
    if outside:
        for g in grads:
            assert not g[:outside].any() and not g[-outside:].any()


@pytest.mark.parametrize("D", [64, 128, 80, 8])
@pytest.mark.parametrize("window,sinks", [(30, 4), (1, 1), (200, 70), (64, 128), (64, 129)])
def test_one_long_sequence(D, window, sinks):
    check([2100], [2100], 4, 2, D, window, sinks)


def test_packed():
    check([1, 333, 0, 1500, 17, 128, 900], [1, 333, 0, 1500, 17, 128, 900], 8, 2, 64, 100, 5)
    check([700, 40], [700, 40], 6, 1, 128, 32, 3, outside=7)
    check([900, 300, 0], [1200, 0, 50], 4, 4, 64, 50, 20)          # queries of no keys, keys of no queries
    check([1300, 100], [600, 900], 4, 1, 64, 40, 90)               # fewer keys than queries, and more


def test_batches():
    check([800] * 3, [800] * 3, 4, 1, 64, 64, 4, batch=True)
    check([500] * 2, [1100] * 2, 4, 2, 128, 64, 33, batch=True)


def test_many_sequences():
    """Tiles enough that the rest is in one part."""
    lens = [700] + [20 + i % 7 for i in range(62)] + [90]
    check(lens, lens, 16, 16, 64, 16, 4)


def test_one_key_is_exact():
    """A row that sees one key gives its value, and dS, dQ and dK of it are zeros: dP and
    do . o are the same sum, but for the order (2 D steps of binary32 of its terms)."""
    say("one key")
    for D in (64, 128):
        q, k, v, do = (rand(i, 200, 2, D).requires_grad_(i < 4) for i in range(1, 5))
        o = attention(q, k, v, window=1)
        assert torch.equal(o, v)
        dq, dk, dv = torch.autograd.grad(o, (q, k, v), do)
        assert torch.equal(dv, do)
        ds = 2 * 2 * D * 2.0 ** -24 * (do * v).double().abs().sum(-1, keepdim=True) * D ** -0.5
        assert (dq.double().abs() <= 1.01 * ds * k.double().abs()).all() and (dk.double().abs() <= 1.01 * ds * q.double().abs()).all()
