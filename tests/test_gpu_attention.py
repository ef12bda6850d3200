"""Attention on the GPU, against 64 bits: lengths from one on, ragged sequences,
windows and sinks, rows that see nothing, heads and strides; gradients, also against
differences; replays, repeated calls."""

import pytest
import torch

import attention_model as model
from gpu_util import say
from paper_2609_02846_amd.attention import attention, attention_forward

pytestmark = pytest.mark.gpu


def rand(seed, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def starts(lens):
    return torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=torch.int32).cuda()


def check(q_lens, k_lens, Hq, Hk, D, dtype, train, seed=0, spread=1.5, **mask):
    say("attention", q_lens, k_lens, Hq, Hk, D, dtype, train, mask)
    q = (spread * rand(seed, sum(q_lens), Hq, D)).to(dtype).requires_grad_(train)
    k, v = (rand(seed + i, sum(k_lens), Hk, D, dtype=dtype).requires_grad_(train) for i in (1, 2))
    scale = D ** -0.5
    o = attention(q, k, v, starts(q_lens), starts(k_lens), **mask)
    do = rand(seed + 3, *o.shape, dtype=dtype)
    grads = torch.autograd.grad(o, (q, k, v), do) if train else None
    _, lse = attention_forward(q.detach(), k.detach(), v.detach(), starts(q_lens), starts(k_lens), lse=True, **mask)
    a = b = 0
    for L, S in zip(q_lens, k_lens):
        rows, keys = slice(a, a + L), slice(b, b + S)
        want = model.Sequence(q[rows].detach(), k[keys].detach(), v[keys].detach(), scale, **mask)
        name = f"{L} x {S}"
        model.within(o[rows].detach(), want.o.transpose(0, 1), want.o_bound().transpose(0, 1), name + " o")
        some = want.lse > -float("inf")
        assert torch.equal(lse[:, rows] > -float("inf"), some)
        err = (lse[:, rows].double() - want.lse)[some].abs()
        assert (err <= (want.rel + model.F * want.lse.abs().unsqueeze(-1)).squeeze(-1)[some]).all(), name + " lse"
        if train:
            w, bound = want.gradients(do[rows])
            model.within(grads[0][rows], w[0], bound[0], name + " dq")
            model.within(grads[1][keys], w[1], bound[1], name + " dk")
            model.within(grads[2][keys], w[2], bound[2], name + " dv")
        a, b = a + L, b + S


@pytest.mark.parametrize("D", [128, 64, 8, 80, 96])
def test_lengths(D):
    for i, L in enumerate([1, 2, 31, 33, 63, 64, 65, 127, 128, 129, 200, 300]):
        check([L], [L], 2, 1, D, torch.bfloat16, True, seed=i)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_more_keys_than_queries_and_fewer(dtype):
    for i, (L, S) in enumerate([(1, 500), (7, 130), (128, 257), (100, 1), (130, 65), (64, 0), (1, 0), (200, 130), (777, 1000)]):
        check([L], [S], 4, 2, 64 if i % 2 else 128, dtype, dtype == torch.bfloat16, seed=i)
        check([L], [S], 4, 2, 64, dtype, dtype == torch.bfloat16, seed=i, causal=False)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (64, 0), (64, 64), (100, 70), (128, 4), (300, 0), (1000, 5), (10 ** 6, 10 ** 6)])
def test_windows_and_sinks(window, sinks):
    check([400], [400], 2, 1, 64, torch.bfloat16, True, window=window, sinks=sinks)
    check([130, 1, 333], [333, 200, 333], 3, 3, 128, torch.bfloat16, True, window=window, sinks=sinks)
    check([100], [40], 2, 2, 64, torch.bfloat16, True, window=window, sinks=sinks)      # rows that see nothing


def test_ragged():
    check([1, 333, 0, 5, 129, 128], [1, 333, 0, 5, 129, 128], 6, 2, 64, torch.bfloat16, True)
    check([0, 0, 3], [0, 5, 3], 2, 1, 128, torch.bfloat16, True)
    lens = [(i * 37) % 11 for i in range(150)]       # more sequences than a wave has lanes
    check(lens, lens, 2, 1, 64, torch.bfloat16, True)
    check(lens, [n + i % 3 for i, n in enumerate(lens)], 2, 1, 64, torch.float16, False)


@pytest.mark.parametrize("heads", [(1, 1), (8, 1), (32, 8), (9, 3), (5, 5), (12, 4)])
def test_heads(heads):
    check([150], [150], *heads, 64, torch.bfloat16, True)


def test_sharp_and_flat_rows():
    """Scores over 400 wide (one key has all the weight), rising along the keys, and
    all alike."""
    check([300], [300], 2, 1, 128, torch.bfloat16, True, spread=30.0)
    L, D = 400, 64
    q, v = torch.ones(L, 1, D, dtype=torch.bfloat16).cuda(), rand(1, L, 1, D)
    for slope in (-0.5, 0.0, 0.5):
        k = (torch.arange(L).view(L, 1, 1) * slope * torch.ones(L, 1, D)).to(torch.bfloat16).cuda()
        want = model.Sequence(q, k, v, D ** -0.5)
        o = attention(q, k, v)
        model.within(o, want.o.transpose(0, 1), want.o_bound().transpose(0, 1), slope)


def test_batches_and_strides():
    x = rand(0, 3, 70, 6, 64)
    q, k, v = x[:, :, :4], x[:, :, 4:5], x[:, :, 5:]
    want = attention(q.contiguous(), k.contiguous(), v.contiguous(), window=20, sinks=2)
    assert torch.equal(attention(q, k, v, window=20, sinks=2), want)
    for b in range(3):
        assert torch.equal(attention(q[b], k[b], v[b], window=20, sinks=2), want[b])
    s = starts([70, 70, 70])
    assert torch.equal(attention(q.reshape(210, 4, 64), k.reshape(210, 1, 64), v.reshape(210, 1, 64), s, window=20, sinks=2),
                       want.view(210, 4, 64))
    hnd = q.transpose(1, 2).contiguous().transpose(1, 2)        # heads apart
    assert torch.equal(attention(hnd, k, v, window=20, sinks=2), want)
    odd = torch.empty(q.numel() + 1, dtype=q.dtype, device="cuda")[1:].view(q.shape).copy_(q)
    assert torch.equal(attention(odd, k, v, window=20, sinks=2), want)
    wide = k[:, :1].expand(3, 70, 1, 64)                        # one key for all tokens
    assert torch.equal(attention(q, wide, v), attention(q, wide.contiguous(), v))
    leaf = v[:, :, :].detach().requires_grad_()
    o = attention(q, k, leaf.expand(3, 70, 1, 64))
    o.float().sum().backward()
    assert leaf.grad.shape == leaf.shape


def test_tokens_of_no_sequence():
    q, k, v = (rand(i, 300, 2, 64).requires_grad_() for i in range(3))
    s = torch.tensor([10, 100, 250], dtype=torch.int32).cuda()
    o = attention(q, k, v, s)
    do = rand(4, 300, 2, 64)
    grads = torch.autograd.grad(o, (q, k, v), do)
    inner = [t[10:250].detach().requires_grad_() for t in (q, k, v)]
    oi = attention(*inner, starts([90, 150]))
    gi = torch.autograd.grad(oi, inner, do[10:250])
    for t, u in zip((o, *grads), (oi, *gi)):
        assert torch.equal(t[10:250], u) and not t[:10].any() and not t[250:].any()
    _, lse = attention_forward(q.detach(), k.detach(), v.detach(), s, lse=True)
    assert (lse[:, 250:] == -float("inf")).all() and (lse[:, :10] == -float("inf")).all()
    # what lies outside does not matter, whatever it is
    bad = [t.detach().clone() for t in (q, k, v)]
    for t in bad:
        t[:10], t[250:] = float("nan"), float("inf")
    assert torch.equal(attention(*bad, s), o)
    # starts past the tokens are kept within them
    wild = torch.tensor([-7, 2 ** 31 - 2, 2 ** 31 - 1], dtype=torch.int32).cuda()
    one = attention(q.detach(), k.detach(), v.detach(), wild)
    assert torch.equal(one, attention(q.detach(), k.detach(), v.detach()))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 128, 40])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_seen_does_not_matter(bad, D, dtype):
    """Keys and values that are not finite change the rows that see them only."""
    L, H = 200, 2
    q, k, v = (rand(i, L, n, D, dtype=dtype) for i, n in ((0, H), (1, 1), (2, 1)))
    for window, sinks, at in ((0, 0, [70]), (0, 0, [199]), (0, 0, [64, 130]), (50, 0, [0, 60]), (20, 70, [10, 66, 150]), (30, 3, [2, 5])):
        want = attention(q, k, v, window=window, sinks=sinks)
        sees = model.visible(L, L, True, window, sinks)[:, at].any(1)
        for where in ("k", "v", "kv"):
            k2, v2 = k.clone(), v.clone()
            for t, n in ((k2, "k"), (v2, "v")):
                if n in where:
                    t[at, 0, D // 2] = bad
            o = attention(q, k2, v2, window=window, sinks=sinks)
            assert torch.equal(o[~sees], want[~sees]), (window, sinks, at, where)
            if where == "v":
                assert not torch.isfinite(o[sees]).all(-1).any(), (window, sinks, at)


def test_differences():
    """The gradient along a direction against a difference of the 64-bit model, whose
    own gradient the kernel is held to above: the model's formula itself."""
    torch.manual_seed(1)
    q, k, v = (torch.randn(9, 2, 8).double() for _ in range(3))
    do = torch.randn(9, 2, 8).double()
    model.U[torch.float64] = model.STEP[torch.float64] = 0.0
    f = lambda q, k, v: (model.Sequence(q, k, v, 0.4, window=5, sinks=1).o.transpose(0, 1) * do).sum()  # noqa: E731
    grads, _ = model.Sequence(q, k, v, 0.4, window=5, sinks=1).gradients(do)
    h = 1e-5
    for i, g in enumerate(grads):
        d = torch.randn_like(g)
        up, down = [[t + s * h * d if j == i else t for j, t in enumerate((q, k, v))] for s in (1, -1)]
        assert abs((f(*up) - f(*down)) / (2 * h) - (g * d).sum()) <= 1e-8 * (1 + d.abs().sum())


def test_same_bits_and_some_gradients():
    q, k, v = (rand(i, 700, 4, 128).requires_grad_() for i in range(3))
    do = rand(5, 700, 4, 128)
    runs = []
    for _ in range(3):
        o = attention(q, k, v, window=200, sinks=3)
        runs.append((o.detach(), *torch.autograd.grad(o, (q, k, v), do)))
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(runs[0], r))
    for i in range(3):
        leaves = [t.detach().requires_grad_(j == i) for j, t in enumerate((q, k, v))]
        g, = torch.autograd.grad(attention(*leaves, window=200, sinks=3), leaves[i], do)
        assert torch.equal(g, runs[0][1 + i])


@pytest.mark.parametrize("mask", [{}, dict(causal=False), dict(window=900, sinks=70), dict(window=3000, sinks=0)])
def test_keys_in_parts(mask):
    """Few queries over many keys: their parts joined, with rows of no sequence and rows
    whose parts see nothing."""
    check([100], [3000], 2, 1, 128, torch.bfloat16, True, **mask)
    check([1], [2049], 4, 2, 64, torch.float16, False, **mask)
    check([130, 0, 3], [2600, 700, 1700], 2, 2, 64, torch.bfloat16, True, **mask)
    check([200], [1100], 1, 1, 80, torch.bfloat16, True, **mask)
    q, k, v = rand(1, 50, 2, 64), rand(2, 4000, 1, 64), rand(3, 4000, 1, 64)
    s, t = torch.tensor([3, 40], dtype=torch.int32).cuda(), torch.tensor([0, 4000], dtype=torch.int32).cuda()
    o, lse = attention_forward(q, k, v, s, t, lse=True, **mask)
    assert not o[:3].any() and not o[40:].any() and (lse[:, 40:] == -float("inf")).all()
    whole = model.Sequence(q[3:40], k, v, 64 ** -0.5, **mask)
    model.within(o[3:40], whole.o.transpose(0, 1), whole.o_bound().transpose(0, 1), "inner")


def test_empty():
    q, k = rand(0, 0, 2, 64).requires_grad_(), rand(1, 5, 2, 64).requires_grad_()
    o = attention(q, k, k.detach().requires_grad_(), starts([0]), starts([5]))
    assert o.shape == (0, 2, 64)
    g, = torch.autograd.grad(o, k, torch.zeros_like(o))
    assert g.shape == k.shape and not g.any()
    e = rand(0, 0, 7, 2, 64)
    assert attention(e, e, e).shape == e.shape


def test_replays_of_a_captured_step():
    data = [rand(i, 300, 2, 64) for i in range(3)]
    held = [t.clone() for t in data]
    s, do = starts([100, 200]), rand(9, 300, 2, 64)

    def step(tensors):
        leaves = [t.detach().requires_grad_() for t in tensors]
        o = attention(*leaves, s, window=50, sinks=2)
        return (o.detach(), *torch.autograd.grad(o, leaves, do))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):                    # no call came before
        out = step(held)
    for i in range(4):
        for t, d in zip(held, data):
            t.copy_(d * (i + 1) / 2)
        s.copy_(starts([100, 200] if i % 2 else [17, 283]))
        want = step(held)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i


def test_two_streams():
    data = [[rand(10 * s + i, 500, 4, 64) for i in range(3)] for s in range(2)]
    want = [attention(*d) for d in data]
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(attention(*data[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in range(2) for o in got[i])
