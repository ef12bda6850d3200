"""Rows whose seen keys all score -inf, as keys of infinities make them: their softmax is 0 / 0
and they are NaN, while a row that sees nothing is zeros and a key of -inf among others
weighs nothing."""

import pytest
import torch

import attention_model as model
from gpu_util import say
from paper_2609_02846_amd.attention import attention, attention_forward, paged_attention

pytestmark = pytest.mark.gpu


def inputs(L, S, H, Hk, D, dtype, bad, seed=0):
    """Queries of positive first elements; keys `bad` start with -inf."""
    g = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn(n, h, D, generator=g).to(dtype).cuda() for n, h in ((L, H), (S, Hk), (S, Hk)))
    q[..., 0] = 1.0
    k[bad, :, 0] = -float("inf")
    return q, k, v


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 128, 40])
def test_rows_of_infinite_scores_alone(D, dtype):
    for L, S in ((1, 1), (5, 5), (70, 70), (200, 200), (3, 3000), (100, 2600)):       # (the last two in parts)
        say("all", L, S, D, dtype)
        o, lse = attention_forward(*inputs(L, S, 2, 1, D, dtype, slice(None)), lse=True)
        assert torch.isnan(o).all(), (L, S)
        # (heads of 40 are padded, which makes the score -inf + 0 inf, a NaN)
        assert (torch.isnan(lse) if D == 40 else lse == -float("inf")).all(), (L, S)
    for L, S in ((5, 3), (200, 130)):
        say("some see nothing", L, S, D, dtype)
        o = attention(*inputs(L, S, 2, 1, D, dtype, slice(None)))
        assert not o[:L - S].any() and torch.isnan(o[L - S:]).all()
    q, k, v = inputs(50, 2000, 2, 1, D, dtype, slice(None))
    s, t = torch.tensor([3, 40], dtype=torch.int32).cuda(), torch.tensor([0, 2000], dtype=torch.int32).cuda()
    o = attention(q, k, v, s, t)
    assert torch.isnan(o[3:40]).all() and not o[:3].any() and not o[40:].any()


@pytest.mark.parametrize("D", [64, 128])
def test_a_key_of_minus_infinity_weighs_nothing(D):
    for L, n, first in ((70, 70, 1), (200, 200, 65), (100, 3000, 1500)):
        say("first keys", L, n, first)
        q, k, v = inputs(L, n, 2, 1, D, torch.bfloat16, slice(0, first))
        o = attention(q, k, v)
        rows = max(0, L - (n - first))               # those whose keys are all of them
        assert torch.isnan(o[:rows]).all()
        want = model.Sequence(q[rows:], k[first:], v[first:], D ** -0.5)
        model.within(o[rows:], want.o.transpose(0, 1), want.o_bound().transpose(0, 1), (L, n, first))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_paged(dtype):
    lens, page = [1, 40, 0, 1500, 33, 700], 16       # 1500: in parts
    for bad in (lens, [0, 0, 0, 0, 32, 600]):
        say("paged", bad)
        need = [-(-n // page) for n in lens]
        kc, vc = (torch.zeros(sum(need), page, 2, 64, dtype=dtype, device="cuda") for _ in range(2))
        table, at, seqs = torch.zeros(len(lens), max(need), dtype=torch.int32), 0, []
        for b, n in enumerate(lens):
            seqs.append(inputs(1, n, 4, 2, 64, dtype, slice(0, bad[b]), seed=b))
            table[b, :need[b]] = torch.arange(at, at + need[b])
            for c, t in zip((kc, vc), seqs[-1][1:]):
                c[at:at + need[b]].view(-1, 2, 64)[:n] = t
            at += need[b]
        q = torch.cat([s[0] for s in seqs])
        o = paged_attention(q, kc, vc, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
        for b, n in enumerate(lens):
            if n == 0:
                assert not o[b].any()
            elif bad[b] == n:
                assert torch.isnan(o[b]).all(), (b, n)
            else:
                want = model.Sequence(seqs[b][0], *(t[bad[b]:] for t in seqs[b][1:]), 64 ** -0.5)
                model.within(o[b:b + 1], want.o.transpose(0, 1), want.o_bound().transpose(0, 1), (b, n))
