"""What the forward pass keeps of its output's rounding for the gradients, and dS as two
numbers: pinned where the rest of the arithmetic is exact.

With queries of zeros every weight of a row is 1 / n, P itself 1, and values and output
gradients of a few bits make all products and sums exact.  With all keys alike dQ =
scale k sum(dS) is 0, as a row's dS add up to nothing, and what the kernel gives instead
is the error of delta = do . o and of dS alone."""

import pytest
import torch

import attention_model as model

F, U = model.F, model.U[torch.bfloat16]
#            queries, keys, mask; the last three with the keys in parts
CASES = [(1, 1, {}), (3, 3, {}), (40, 40, {}), (200, 200, {}), (130, 300, dict(window=90, sinks=5)), (100, 100, dict(causal=False)),
         (100, 3000, {}), (9, 2500, dict(causal=False)), (50, 2600, dict(window=2000, sinks=7))]


def inputs(L, S, H, Hk, D, seed=0):
    """q of zeros, k all alike, v and do of multiples of 1/8 below 2."""
    g = torch.Generator().manual_seed(seed)
    eighths = lambda n, h: (torch.randint(-15, 16, (n, h, D), generator=g) / 8).to(torch.bfloat16)  # noqa: E731
    q = torch.zeros(L, H, D, dtype=torch.bfloat16)
    k = torch.randn(1, Hk, D, generator=g).to(torch.bfloat16).expand(S, Hk, D).contiguous()
    return q, k, eighths(S, Hk) + 0.5, eighths(L, H)


def exact(v, do, H, mask):
    """(o, t, delta, P, n) in 64 bits, heads first; t = do . v."""
    L, S = do.shape[0], v.shape[0]
    see = model.visible(L, S, device=v.device, **mask)
    n = see.sum(-1, keepdim=True).double()
    v = v.double().transpose(0, 1).repeat_interleave(H // v.shape[1], 0)
    do = do.double().transpose(0, 1)
    p = see / n
    o = see.double() @ v / n                         # (the sums are exact; the weights are not)
    return o, do @ v.transpose(1, 2), (do * o).sum(-1, keepdim=True), p, n


def o_bounds(o):
    """Of o and of o + o_rest: a quotient (2.5 steps of binary32) and a product, together less
    than 2^-21; the rounding of o; that of what it left."""
    return (U + 2.0 ** -21) * o.abs(), (U * U * (1 + U) + 2.0 ** -21) * o.abs()


def dq_bound(do, k, o, t, delta, p, n, scale):
    """How far dQ may be from 0.  delta: that of o + o_rest, and a sum of D terms; dS: its
    difference and its product with P (off by less than 2^-17, which all keys share: log n and
    its exponential, 12 steps of 2^-21), two numbers that leave U^2 of it, and the sums of
    two products over the keys; dQ's own rounding."""
    D = do.shape[-1]
    do = do.double().transpose(0, 1).abs()
    err = (do * o_bounds(o)[1]).sum(-1, keepdim=True) + (D + 2) * F * (do * o.abs()).sum(-1, keepdim=True)
    ds = p * (1 + 2.0 ** -17) * (err + (U * U * (1 + U) + (2 * n + 18) * F) * (t - delta).abs())
    k = k[0].double().abs().repeat_interleave(do.shape[0] // k.shape[1], 0)[:, None]
    return (scale * (1 + 2 * U) * ds.sum(-1, keepdim=True) * k).transpose(0, 1) + 1e-30


@pytest.mark.parametrize("case", [2, 3, 4, 5, 6])
def test_the_bound_sees_what_is_left_out(case):
    """dQ from o as it was rounded, and with dS in one number, would be beyond the bound."""
    L, S, mask = CASES[case]
    H, Hk, D = 4, 2, 16
    q, k, v, do = inputs(L, S, H, Hk, D)
    o, t, delta, p, n = exact(v, do, H, mask)
    bound = dq_bound(do, k, o, t, delta, p, n, 0.25)
    wide = k.double().transpose(0, 1).repeat_interleave(2, 0)
    rounded = lambda x: x.to(torch.bfloat16).double()  # noqa: E731
    dod = do.double().transpose(0, 1)
    two = lambda s: rounded(s) + rounded(s - rounded(s))  # noqa: E731
    rest = rounded(o) + rounded(o - rounded(o))
    dq = lambda o, split: (0.25 * split(p * (t - (dod * o).sum(-1, keepdim=True))) @ wide).transpose(0, 1)  # noqa: E731
    ratio = lambda x: (x.abs() / bound).max().item()  # noqa: E731
    assert ratio(dq(rest, two)) <= 1.0
    assert ratio(dq(rounded(o), two)) > 1.5
    if S <= 300:                                     # (over thousands of keys their roundings cancel)
        assert ratio(dq(rest, rounded)) > 1.5
    assert ((rounded(o) - o).abs() > 4 * o_bounds(o)[1]).any() and ((rest - o).abs() <= o_bounds(o)[1]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("L,S,mask", CASES)
@pytest.mark.parametrize("D", [16, 64, 80, 128])
def test_on_the_gpu(L, S, mask, D):
    from gpu_util import say
    from paper_2609_02846_amd import AttentionC, load_library
    from paper_2609_02846_amd.attention import attention, attention_forward

    say("rest", L, S, mask, D)
    H, Hk = 4, 2
    q, k, v, do = (t.cuda() for t in inputs(L, S, H, Hk, D, seed=D))
    parts = load_library().ue5m3_attention_scratch(AttentionC(q_tokens=L, k_tokens=S, sequences=1, q_heads=H, kv_heads=Hk, dim=D, causal=1,
                                                              window=mask.get("window", 0), sinks=mask.get("sinks", 0)))
    assert (parts > 0) == (S > 1000)
    want, t, delta, p, n = exact(v, do, H, mask)
    o, lse, rest = attention_forward(q, k, v, lse=True, _rest=True, **mask)
    whole, with_rest = o_bounds(want)
    heads_first = lambda x: x.double().transpose(0, 1)  # noqa: E731
    model.within(heads_first(o), want, whole + 1e-30, "o")
    model.within(heads_first(o) + heads_first(rest), want, with_rest + 1e-30, "o and its rest")
    leaves = [x.detach().requires_grad_() for x in (q, k, v)]
    dq, = torch.autograd.grad(attention(*leaves, **mask), leaves[:1], do)
    model.within(dq, torch.zeros_like(dq, dtype=torch.float64), dq_bound(do, k, want, t, delta, p, n, D ** -0.5), "dq")
