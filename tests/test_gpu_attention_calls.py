"""Calls of the operators between the projections as programs make them: one tensor in
several places, broadcast heads and gradients, activation checkpointing, host threads,
two captured graphs, caches that autograd has saved, batches of nothing."""

import threading

import pytest
import torch
from torch.utils.checkpoint import checkpoint

from gpu_util import say
from paper_2609_02846_amd.attention import attention, paged_attention
from paper_2609_02846_amd.paged import PagedCache, copy_pages
from paper_2609_02846_amd.rotary import qk_norm_rope, qk_norm_rope_append, rotary_frequencies
from paper_2609_02846_amd.sublayer import PreNormAttention

pytestmark = pytest.mark.gpu


def rand(seed, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def test_one_tensor_as_all_three():
    """The gradient is the sum of the three parts', in 16 bits as autograd adds them."""
    say("one tensor")
    x = rand(1, 2, 70, 3, 64).requires_grad_()
    do = rand(2, *x.shape)
    g, = torch.autograd.grad(attention(x, x, x), x, do)
    leaves = [x.detach().clone().requires_grad_() for _ in range(3)]
    parts = [p.double() for p in torch.autograd.grad(attention(*leaves), leaves, do)]
    # (two sums, each off by half a step of at most the magnitudes' sum)
    size = sum(p.abs() for p in parts)
    assert ((g.double() - sum(parts)).abs() <= 2.01 * 2.0 ** -8 * size).all()


def test_broadcast_heads_and_gradients():
    say("broadcast")
    q, k = rand(1, 90, 4, 64).requires_grad_(), rand(2, 90, 1, 64).requires_grad_()
    wide = k.expand(90, 2, 64)
    o = attention(q, wide, wide)
    want = attention(q, wide.contiguous(), wide.contiguous())
    assert torch.equal(o, want)
    # a sum's gradient is one number, expanded
    got = torch.autograd.grad(o.float().sum(), (q, k), retain_graph=True)
    full = torch.autograd.grad(want, (q, k), torch.ones_like(o))
    again = torch.autograd.grad(o, (q, k), torch.ones_like(o[:1]).expand_as(o))
    for a, b, c in zip(got, full, again):
        assert torch.equal(a, b) and torch.equal(c, b)
    a, b = qk_norm_rope(q, k, freqs=rotary_frequencies(64)[0])
    one = torch.ones((), dtype=torch.bfloat16, device="cuda")
    x = torch.autograd.grad((a, b), (q, k), (one.expand_as(a), one.expand_as(b)), retain_graph=True)
    y = torch.autograd.grad((a, b), (q, k), (torch.ones_like(a), torch.ones_like(b)))
    assert all(torch.equal(s, t) for s, t in zip(x, y))


def test_checkpointed_branch():
    say("checkpoint")
    m, x = PreNormAttention(128, 4, 2, 32, p=0.2), rand(3, 2, 65, 128).requires_grad_()
    leaves, grads = [x, *m.parameters()], []
    for run in (m, lambda t: checkpoint(m, t, use_reentrant=False)):
        torch.manual_seed(11)
        grads.append(torch.autograd.grad(run(x), leaves, rand(4, 2, 65, 128)))
    assert all(torch.equal(a, b) for a, b in zip(*grads))


def test_host_threads_on_one_stream():
    say("threads")
    data = [[rand(10 * i + j, 60, 8, 128) for j in range(3)] for i in range(4)]
    keys = [rand(50 + i, 3000, 8, 128) for i in range(4)]
    want = [(attention(*d), attention(d[0], k, k, causal=False)) for d, k in zip(data, keys)]
    got = [[] for _ in data]

    def work(i):
        for _ in range(20):
            got[i].append((attention(*data[i]), attention(data[i][0], keys[i], keys[i], causal=False)))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert len(g) == 20 and all(torch.equal(a, b) for pair in g for a, b in zip(pair, w))


def test_two_graphs_share_nothing():
    """Keys in parts, whose sums lie in scratch memory: each graph has its own."""
    say("two graphs")
    data = [[rand(10 * i, 40, 8, 128), *(rand(10 * i + j, 4000, 8, 128) for j in (1, 2))] for i in range(2)]
    want = [attention(*d) for d in data]
    graphs, outs = [], []
    for d in data:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(attention(*d))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(4):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want)), turn


def test_saved_caches_are_noticed():
    say("saved caches")
    c = PagedCache(1, 4, 16, 2, 64)
    slots = c.extend([c.open()], [20])
    k, v = rand(1, 20, 2, 64), rand(2, 20, 2, 64)
    for change in (lambda: qk_norm_rope_append(None, k, v, *c.layer(0), slots, eps=None),
                   lambda: copy_pages(c.storage, [0], [3], dim=2)):
        w = torch.ones(64, dtype=torch.bfloat16, device="cuda", requires_grad=True)
        y = (c.layer(0)[0] * w).sum()
        change()
        with pytest.raises(RuntimeError, match="inplace"):
            y.backward()


def test_batches_of_nothing():
    say("nothing")
    c = PagedCache(1, 4, 16, 2, 64)
    for n in (0, 3):                                 # no rows, rows of no tokens
        table, lengths = c.tables([c.open() for _ in range(n)])
        assert table.shape == (n, 0)
        o = paged_attention(rand(n, n, 6, 64), *c.layer(0), table, lengths)
        assert o.shape == (n, 6, 64) and not o.any()
    assert c.extend([], []).shape == (0,) and c.extend([0], [0]).shape == (0,)
    e = rand(0, 0, 2, 64)
    before = c.storage.clone()
    assert qk_norm_rope_append(e, e, e, *c.layer(0), c.extend([], [])).shape == (0, 2, 64)
    copy_pages(c.storage, [], [], dim=2)
    assert torch.equal(c.storage, before)
    m = PreNormAttention(128, 4, 2, 32)
    x = rand(0, 0, 128).requires_grad_()
    y = m(x)
    assert y.shape == (0, 128)
    y.sum().backward()
    assert x.grad.shape == (0, 128) and not m.q_weight.grad.any() and not m.qkv.weight.grad.any()


def test_offsets_past_32_bits():
    """Tokens 8 MB apart: the same bits as of dense ones."""
    say("far apart")
    T, step = 600, 1 << 22                           # the last token is 5 GB from the first

    def apart(t):
        store = torch.empty((T - 1) * step + t[0].numel(), dtype=t.dtype, device="cuda")
        far = store.as_strided(t.shape, (step, t.shape[2], 1))
        return far.copy_(t)
    dense = [rand(1, T, 4, 64), rand(2, T, 2, 64), rand(3, T, 2, 64)]
    do, f = rand(4, T, 4, 64), rotary_frequencies(64)[0]
    want = got = None
    for tensors in (dense, [apart(t) for t in dense]):
        q, k, v = (t.detach().requires_grad_() for t in tensors)
        a, b = qk_norm_rope(q, k, freqs=f)
        o = attention(q, k, v, window=100, sinks=3)
        got = [a, b, o, *torch.autograd.grad(o, (q, k, v), do), *torch.autograd.grad((a, b), (q, k), (do, dense[1]))]
        if want is None:
            want = got
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_another_stream():
    """Forward and backward pass on a stream of their own, its memory used again at once."""
    say("another stream")
    x = [rand(i, 400, 4, 64).requires_grad_() for i in range(3)]
    do = rand(9, 400, 4, 64)

    def step():
        a, b = qk_norm_rope(x[0], x[1], freqs=f)
        return torch.autograd.grad(attention(a, b, x[2], window=64, sinks=2), x, do)
    f = rotary_frequencies(64)[0]
    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = [step() for _ in range(10)]
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))


def test_a_branch_cast_with_its_model():
    """The rotation is that of the frequencies in 32 bits."""
    say("cast")
    a, x = PreNormAttention(128, 4, 2, 32).eval(), rand(5, 1, 50, 128)
    positions = torch.arange(50, device="cuda") + 100000
    want = a(x, positions=positions)
    assert torch.equal(a.to(torch.bfloat16)(x, positions=positions), want)
