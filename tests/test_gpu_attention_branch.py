"""The attention branch: equal to the separate operators, bit for bit, forward and
backward, in packed sequences; prompts and single tokens over a cache."""

import pytest
import torch

from gpu_util import say
from paper_2609_02846_amd.attention import attention, paged_attention
from paper_2609_02846_amd.dropout import dropout
from paper_2609_02846_amd.fp8 import fp8_linear
from paper_2609_02846_amd.norm import layer_norm
from paper_2609_02846_amd.paged import PagedCache
from paper_2609_02846_amd.rotary import packed_positions, qk_norm_rope, qk_norm_rope_append, rotary_frequencies
from paper_2609_02846_amd.sublayer import PreNormAttention

pytestmark = pytest.mark.gpu


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()


def starts(*at):
    return torch.tensor(at, dtype=torch.int32).cuda()


def test_packed_positions():
    assert packed_positions(starts(0, 3, 3, 7), 9).tolist() == [0, 1, 2, 0, 1, 2, 3, 0, 1]
    assert packed_positions(starts(2, 4), 5)[2:4].tolist() == [0, 1]


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("window", [0, 20])
def test_equals_the_separate_calls(packed, window):
    say("attention branch", packed, window)
    m = PreNormAttention(192, 6, 2, 64, p=0.2, seed=4, layer_id=3, window=window, sinks=2, rotary=rotary_frequencies(32, factor=2.0))
    with torch.no_grad():
        m.q_weight.copy_(1 + 0.1 * rand(1, 64)), m.k_weight.copy_(1 + 0.1 * rand(2, 64))
    x = (rand(3, 100, 192) if packed else rand(3, 4, 25, 192)).requires_grad_()
    s = starts(0, 30, 31, 100) if packed else None
    y, dy = m(x, s), rand(5, *x.shape)
    leaves = [x, *m.parameters()]
    got = torch.autograd.grad(y, leaves, dy)
    h = layer_norm(x, m.norm.weight, m.norm.bias, m.norm.eps)
    qkv = fp8_linear(h, m.qkv.weight).view(*x.shape[:-1], 10, 64)
    pos = packed_positions(s, 100) if packed else None
    q, k = qk_norm_rope(qkv[..., :6, :], qkv[..., 6:8, :], m.q_weight, m.k_weight, pos, m.freqs)
    o = attention(q, k, qkv[..., 8:, :], s, window=window, sinks=2)
    want = dropout(fp8_linear(o.reshape(*x.shape[:-1], 384), m.out.weight), 0.2, 4, 3, residual=x)
    assert torch.equal(y, want)
    for p, q in zip(got, torch.autograd.grad(want, leaves, dy)):
        assert torch.equal(p, q)


def test_prompt_and_tokens():
    m = PreNormAttention(256, 4, 2, 64, window=50, sinks=3).eval()
    for layer in (m.qkv, m.out):
        layer.freeze()
    x = rand(7, 91, 256)
    c = PagedCache(1, 20, 16, 2, 64)
    kc, vc = c.layer(0)
    a, b = c.open(), c.open()
    s = starts(0, 60, 90)
    with torch.no_grad():
        y = m.prompt(x[:90], kc, vc, c.extend([a, b], [60, 30]), s)
        assert torch.equal(y, m(x[:90], s))
        token = torch.stack([x[90], x[7]])
        slots = c.extend([a, b], [1, 1])
        table, lengths = c.tables([a, b])
        got = m.token(token, kc, vc, slots, table, lengths)
        before = kc.clone(), vc.clone()
        q, k, v = m.qkv(m.norm(token)).view(2, 8, 64).split([4, 2, 2], dim=1)
        q = qk_norm_rope_append(q, k, v, kc, vc, slots, m.q_weight, m.k_weight, lengths - 1, m.freqs)
        want = token + m.out(paged_attention(q, kc, vc, table, lengths, window=50, sinks=3).view(2, 256))
        assert torch.equal(got, want) and torch.equal(kc, before[0]) and torch.equal(vc, before[1])
    with pytest.raises(RuntimeError, match="no gradients"):
        paged_attention(q.requires_grad_(), kc, vc, table, lengths)


def test_a_captured_training_step():
    """Every replay of a captured step equals an eager one.  (No eager graph of the
    parameters lives while it is captured: each step hands its gradients on.)"""
    m = PreNormAttention(128, 2, 1, 64, p=0.0)
    x, dy = rand(1, 1, 70, 128), rand(2, 1, 70, 128)
    held, leaves = x.clone(), list(m.parameters())

    def step(t):
        t = t.detach().requires_grad_()
        y = m(t)
        return (y.detach(), *torch.autograd.grad(y, [t, *leaves], dy))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(held)                                   # the linears' and the norm's workspaces on this stream
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step(held)
    for i in range(3):
        held.copy_(x * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        want = step(held.clone())
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want)), i
