"""Attention, its gradients, paged attention and the rotation of tensors with one token or
one head, at pitches that a tensor of more could not have: as of dense ones."""

import pytest
import torch

from gpu_util import say
from paper_2609_02846_amd.attention import attention, paged_attention
from paper_2609_02846_amd.rotary import qk_norm_rope, qk_norm_rope_append, rotary_frequencies

pytestmark = pytest.mark.gpu


def rand(seed, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def one_token(seed, heads, pitch):
    return rand(seed, 4, heads, pitch)[:1, :, :64]


@pytest.mark.parametrize("pitch", [132, 100, 72])
def test_one_token(pitch):
    say("one token", pitch)
    q, k, v = (one_token(i, 1, pitch) for i in range(3))
    assert torch.equal(attention(q, k, v), v)        # (one key: its value)
    many = [rand(9 + i, 70, 1, 64) for i in range(2)]
    assert torch.equal(attention(q, *many), attention(q.clone(memory_format=torch.contiguous_format), *many))
    wide = one_token(5, 2, pitch)
    assert torch.equal(attention(wide, k, v), v.expand(1, 2, 64))


def test_one_head():
    """Of tensors [tokens, dim, heads], transposed; with gradients."""
    say("one head")
    q, k, v = (rand(i, 90, 64, 1).transpose(1, 2) for i in range(3))
    runs = []
    for make in (lambda t: t.detach(), lambda t: t.detach().clone(memory_format=torch.contiguous_format)):
        leaves = [make(t).requires_grad_() for t in (q, k, v)]
        o = attention(*leaves, window=40, sinks=2)
        runs.append((o, *torch.autograd.grad(o, leaves, rand(7, 90, 1, 64))))
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_rotation():
    say("rotation")
    f = rotary_frequencies(64)[0]
    q, k = one_token(1, 1, 132), one_token(2, 1, 100)
    dense = [t.clone(memory_format=torch.contiguous_format) for t in (q, k)]
    at = torch.tensor([7]).cuda()
    for a, b in zip(qk_norm_rope(q, k, positions=at, freqs=f), qk_norm_rope(*dense, positions=at, freqs=f)):
        assert torch.equal(a, b)


def test_paged():
    """One row, one head, one page: none of their strides reaches anything."""
    say("paged")
    store = rand(3, 2, 4, 16 * 64 + 4)
    kc, vc = (store[i, :1, :16 * 64].view(1, 16, 1, 64) for i in range(2))
    for i, c in enumerate((kc, vc)):
        c.copy_(rand(20 + i, 1, 16, 1, 64))
    kc, vc = (c.as_strided(c.shape, (1028, 64, 3, 1)) for c in (kc, vc))
    q = one_token(4, 1, 132)
    table, lengths = torch.zeros(1, 1, dtype=torch.int32).cuda(), torch.tensor([11], dtype=torch.int32).cuda()
    want = paged_attention(q.clone(memory_format=torch.contiguous_format), *(c.clone(memory_format=torch.contiguous_format) for c in (kc, vc)),
                           table, lengths)
    assert torch.equal(paged_attention(q, kc, vc, table, lengths), want)
    new = one_token(6, 1, 132)
    qk_norm_rope_append(None, new, new, kc, vc, torch.tensor([11]).cuda(), eps=None)
    assert torch.equal(kc[0, 11], new[0]) and torch.equal(vc[0, 11], new[0])
