"""Norms and rotation of queries and keys on the GPU, against 64 bits: values,
gradients (also against differences), types, layouts, strides, positions; the
serving form's slots."""

import pytest
import torch

import attention_model as model
from gpu_util import say
from paper_2609_02846_amd.rotary import qk_norm_rope, qk_norm_rope_append, rotary_frequencies

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]
# tokens, query heads, key-value heads, head size, pairs
SHAPES = [(1, 32, 8, 128, 64), (3, 1, 1, 1, 0), (5, 2, 1, 2, 1), (17, 9, 3, 80, 20), (33, 3, 1, 50, 25), (64, 4, 2, 256, 128),
          (70, 6, 2, 96, 24), (129, 5, 5, 100, 12), (9, 7, 1, 64, 32), (31, 2, 2, 32, 8), (12, 3, 3, 255, 127), (7, 1, 1, 64, 3)]


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def packed(seed, T, Hq, Hk, D, dtype):
    """Queries, keys and values as views of one projection's output."""
    x = (rand(seed, T, Hq + 2 * Hk, D) * (1 + 5 * (rand(seed + 1, T, 1, 1) > 1))).to(dtype).cuda()
    return x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_values_and_gradients(dtype, interleaved):
    for i, (T, Hq, Hk, D, P) in enumerate(SHAPES):
        for norm in (True, False) if P else (True,):
            wt = torch.float32 if i % 3 == 0 else dtype
            say("rope", dtype, interleaved, T, Hq, Hk, D, P, norm)
            q, k, _ = (t.detach().requires_grad_() for t in packed(10 * i, T, Hq, Hk, D, dtype))
            w = [(1 + 0.2 * rand(10 * i + j, D)).to(wt).cuda().requires_grad_() if norm and i != 4 else None for j in (3, 4)]
            freqs = rotary_frequencies(2 * P, 10000.0)[0] if P else None
            positions = (torch.arange(T) * 977 + i * 100003).cuda()
            eps, amp = 1e-6 if norm else None, 1.25 if P else 1.0
            gq, gk = rand(10 * i + 5, T, Hq, D).to(dtype).cuda(), rand(10 * i + 6, T, Hk, D).to(dtype).cuda()
            out = qk_norm_rope(q, k, *w, positions, freqs, eps=eps, interleaved=interleaved, amplitude=amp)
            leaves = [t for t in (q, k, *w) if t is not None]
            grads = dict(zip(map(id, leaves), torch.autograd.grad(out, leaves, (gq, gk))))
            for x, y, g, weight in zip((q, k), out, (gq, gk), w):
                x64 = x.detach().double().requires_grad_()
                w64 = None if weight is None else weight.detach().double().requires_grad_()
                want, size = model.rope(x64, w64, positions, freqs, eps, interleaved, amp)
                model.within(y.detach(), want.detach(), model.rope_bound(want.detach(), size.detach(), dtype), "y")
                wants = torch.autograd.grad(want, [t for t in (x64, w64) if t is not None], g.double())
                back, bsize = model.rope(g.double(), None, -positions, freqs, None, interleaved, amp)
                if norm:
                    r = 1 / torch.sqrt((x64.detach() ** 2).mean(-1, keepdim=True) + eps)
                    hat = (x64.detach() * r).abs()
                    h = bsize * (1 if weight is None else w64.detach().abs())
                    # g turned back, times w; less hat times a mean of up to 256 products
                    bound = 64 * model.F * r * (h + hat * (h * hat).mean(-1, keepdim=True))
                else:
                    hat, bound = None, 32 * model.F * bsize
                model.within(grads[id(x)], wants[0], bound + model.rounding(wants[0], dtype) + 1e-30, "dx")
                if weight is not None:
                    # at most 4 rows a wave in turn, 4 waves, 1024 workgroups in four chains
                    n = 64 + 4 + 4 + 260
                    bound = n * model.F * (bsize * hat).sum((0, 1)) + model.rounding(wants[1], wt)
                    model.within(grads[id(weight)], wants[1], bound + 1e-30, "dw")


def test_differences():
    """The gradient of fp32 calls against central differences of the call: with step h
    the difference is off by its rounding, 2 x 32 x 2^-24 x size / 2 h, and by h^2 / 6 of a
    third derivative that is below 40 / |x|^2 rms here."""
    torch.manual_seed(0)
    T, Hq, Hk, D, h = 2, 2, 1, 16, 2.0 ** -6
    q, k = torch.randn(T, Hq, D).cuda() + 0.5, torch.randn(T, Hk, D).cuda()
    w, f = (1 + 0.1 * torch.randn(D)).cuda(), rotary_frequencies(16)[0]
    dy = torch.randn(T, Hq, D).cuda()
    pos = torch.tensor([5, 123456]).cuda()
    x = q.clone().requires_grad_()
    y, _ = qk_norm_rope(x, k, w, None, pos, f)
    dx, = torch.autograd.grad(y, x, dy)
    for at in [(0, 0, 0), (1, 1, 7), (1, 0, 15), (0, 1, 8)]:
        e = torch.zeros_like(q)
        e[at] = h
        up, down = (qk_norm_rope(q + s * e, k, w, None, pos, f)[0].double() for s in (1, -1))
        fd = ((up - down) * dy.double()).sum().item() / (2 * h)
        tol = (2 * 32 * model.F * (y.abs() * 2 * dy.abs())[at[0], at[1]].sum().item() / (2 * h)
               + h * h / 6 * 40 * dy[at[0], at[1]].abs().sum().item())
        assert abs(fd - dx[at].item()) <= tol, (at, fd, dx[at].item(), tol)


def test_far_positions():
    """Angles of positions up to 2^31 and below zero, to 2^-24 of a turn or better."""
    f = rotary_frequencies(128, 10.0)[0]
    pos = torch.tensor([2 ** 31, 2 ** 31 - 1, -5, -(2 ** 31), 2 ** 24 + 1, 0, 131071]).cuda()
    k = torch.ones(7, 1, 128).cuda()
    y, _ = qk_norm_rope(k, k, None, None, pos, f, eps=None)
    want, size = model.rope(k.double(), None, pos, f, None, False, 1.0)
    model.within(y, want, model.rope_bound(want, size, torch.float32), "far")
    assert torch.equal(y[5], k[5])


def test_strides_batches_and_default_positions():
    f = rotary_frequencies(32)[0]
    x = rand(1, 3, 20, 6, 32).to(torch.bfloat16).cuda()
    pos = torch.arange(20).cuda()
    want = [qk_norm_rope(x[b, :, :4].contiguous(), x[b, :, 4:].contiguous(), None, None, pos, f) for b in range(3)]
    for q, k in ((x[:, :, :4], x[:, :, 4:]), (x[:, :, :4].transpose(1, 2).contiguous().transpose(1, 2), x[:, :, 4:])):
        for p in (None, pos, pos[None], pos.int()):
            a, b = qk_norm_rope(q, k, None, None, p, f)
            assert a.shape == q.shape and b.shape == k.shape and a.is_contiguous()
            for i in range(3):
                assert torch.equal(a[i], want[i][0]) and torch.equal(b[i], want[i][1])
    odd = torch.empty(20 * 5 * 32 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(20, 5, 32).copy_(x[0, :, :5])
    assert torch.equal(qk_norm_rope(odd, odd, None, None, pos, f)[0], qk_norm_rope(x[0, :, :5], x[0, :, :5], None, None, pos, f)[0])
    # a broadcast input's gradient is the sum over what it was broadcast to
    one = rand(2, 20, 1, 32).cuda().requires_grad_()
    y, z = qk_norm_rope(one.expand(20, 4, 32), one, None, None, pos, f)
    g, = torch.autograd.grad((y, z), one, (torch.ones_like(y), torch.zeros_like(z)))
    s = one.detach().requires_grad_()
    y1, z1 = qk_norm_rope(s, s.detach(), None, None, pos, f)
    g1, = torch.autograd.grad(y1, s, torch.ones_like(y1))
    assert torch.allclose(g, 4 * g1, rtol=2.0 ** -22, atol=0)


def test_one_gradient_and_empty():
    f = rotary_frequencies(64)[0]
    q, k, _ = packed(5, 10, 4, 2, 64, torch.bfloat16)
    for need_q, need_k, need_w in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 0, 1)):
        qq, kk, w = q.detach().requires_grad_(bool(need_q)), k.detach().requires_grad_(bool(need_k)), torch.ones(64).cuda().requires_grad_(bool(need_w))
        a, b = qk_norm_rope(qq, kk, w, None, None, f)
        (a.float().sum() + 2 * b.float().sum()).backward()
        full = [t.detach().requires_grad_() for t in (q, k, w)]
        c, d = qk_norm_rope(*full, None, None, f)
        (c.float().sum() + 2 * d.float().sum()).backward()
        for t, u, need in zip((qq, kk, w), full, (need_q, need_k, need_w)):
            assert (t.grad is None) == (not need) and (not need or torch.equal(t.grad, u.grad))
    e = q[:0].detach().requires_grad_()
    w = torch.ones(64).cuda().requires_grad_()
    a, b = qk_norm_rope(e, k[:0], w, None, None, f)
    assert a.shape == (0, 4, 64) and b.shape == (0, 2, 64)
    g, gw = torch.autograd.grad(a, (e, w), torch.zeros_like(a))
    assert g.shape == e.shape and not gw.any()


@pytest.mark.parametrize("dtype", TYPES)
def test_append(dtype):
    for T, Hq, Hk, D, P, page in [(1, 32, 8, 128, 64, 16), (50, 3, 1, 50, 11, 4), (200, 8, 2, 64, 32, 64), (9, 2, 2, 96, 24, 1)]:
        say("append", dtype, T, Hq, Hk, D, P, page)
        q, k, v = packed(T, T, Hq, Hk, D, dtype)
        f, w = rotary_frequencies(2 * P)[0], (1 + 0.1 * rand(3, D)).to(dtype).cuda()
        pages = -(-T // page) + 3
        pos = torch.arange(T).cuda() + 70
        slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(T))[:T].cuda()
        left_out = slots.clone()
        if T > 4:
            left_out[1], left_out[2], left_out[3] = -1, pages * page, 2 ** 62
        a, b = qk_norm_rope(q, k, w, w, pos, f)
        for hnd in (True, False):
            store = torch.full((2, pages, Hk, page, D) if hnd else (2, pages, page, Hk, D), 7.0, dtype=dtype, device="cuda")
            kc, vc = (store[i].transpose(1, 2) if hnd else store[i] for i in (0, 1))
            got = qk_norm_rope_append(q, k, v, kc, vc, left_out, w, w, pos, f)
            assert torch.equal(got, a)
            wk, wv = torch.full_like(kc, 7.0), torch.full_like(vc, 7.0)
            ok = (left_out >= 0) & (left_out < pages * page)
            wk[left_out[ok] // page, left_out[ok] % page], wv[left_out[ok] // page, left_out[ok] % page] = b[ok], v[ok]
            assert torch.equal(kc, wk) and torch.equal(vc, wv)
            # keys that are ready
            kc.fill_(3.0), vc.fill_(3.0)
            assert qk_norm_rope_append(None, b, v, kc, vc, slots, eps=None) is None
            assert torch.equal(kc[slots // page, slots % page], b) and torch.equal(vc[slots // page, slots % page], v)
            assert (kc == 3).sum() >= (pages * page - T) * Hk * D


def test_replays_of_a_captured_step():
    q, k, _ = packed(8, 300, 8, 2, 64, torch.bfloat16)
    f, w = rotary_frequencies(64)[0], (1 + 0.1 * rand(3, 64)).to(torch.bfloat16).cuda()
    gq, gk = rand(4, 300, 8, 64).to(torch.bfloat16).cuda(), rand(5, 300, 2, 64).to(torch.bfloat16).cuda()

    def step(q, k):
        leaves = [t.detach().requires_grad_() for t in (q, k, w)]
        out = qk_norm_rope(*leaves, None, None, f)
        return (*[t.detach() for t in out], *torch.autograd.grad(out, leaves, (gq, gk)))
    qs, ks = q.contiguous(), k.contiguous()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):                    # no call came before
        held = step(qs, ks)
    for i in range(4):
        qs.copy_(q * (i + 1)), ks.copy_(k + i)
        want = step(qs, ks)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, want)), i
