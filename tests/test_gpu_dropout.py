"""Dropout on the GPU: the mask of every element against the oracle's words,
and values bit for bit."""

import numpy as np
import pytest
import torch

import paper_2609_02846_amd as ue
from gpu_util import say
from oracle import fp8
from paper_2609_02846_amd.dropout import Dropout, dropout

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


def expected(x, p, seed, tid, residual=None, first=0):
    d = int(np.rint(p * 65536))
    keep = fp8.dropout_words(seed, tid, first + np.arange(x.numel())) >= d
    up = np.float32(65536.0 / (65536 - d)) if d < 65536 else np.float32(0)
    f = torch.from_numpy(np.where(keep, x.float().cpu().numpy().reshape(-1) * up, np.float32(0))).view(x.shape)
    if residual is not None:
        f = residual.float().cpu() + f
    return f.to(x.dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_every_element(dtype):
    for i, shape in enumerate([(1,), (7,), (8,), (9, 1), (3, 5, 11), (300, 1357), (64, 2048)]):
        for p in (0.0, 0.1, 0.25, 0.5, 0.999, 1.0, 1e-5):
            say("dropout", dtype, shape, p)
            x = torch.randn(shape, generator=torch.Generator().manual_seed(i)).to(dtype).cuda()
            r = torch.randn(shape, generator=torch.Generator().manual_seed(i + 50)).to(dtype).cuda()
            seed, tid = (0x9E3779B97F4A7C15 * (i + 1)) % 2 ** 64, (i * 0x10001) | 0x80000000
            assert torch.equal(ue.dropout_forward(x, p, seed, tid).cpu(), expected(x, p, seed, tid))
            assert torch.equal(ue.dropout_forward(x, p, seed, tid, r).cpu(), expected(x, p, seed, tid, r))


def test_dropped_values_do_not_matter():
    """What is dropped is replaced: NaN and infinities there give the residual."""
    x = torch.ones(4096, device="cuda")
    keep = ue.dropout_forward(x, 0.5, 3, 1) != 0
    for bad in (float("nan"), float("inf"), -float("inf")):
        v = torch.where(keep, x, torch.full_like(x, bad))
        assert torch.equal(ue.dropout_forward(v, 0.5, 3, 1), 2 * keep.float())
        assert torch.equal(ue.dropout_forward(v, 0.5, 3, 1, residual=x), 1 + 2 * keep.float())
    assert not ue.dropout_forward(torch.full_like(x, float("nan")), 1.0, 3, 1).any()


def test_statistics():
    """Share kept and the mean, within six standard deviations; keys and tensor
    ids give unrelated masks."""
    n, p = 1 << 22, 0.1
    x = torch.ones(n, device="cuda")
    a = ue.dropout_forward(x, p, 1, 0)
    d = round(p * 65536)
    q = d / 65536
    kept = (a != 0).double().mean().item()
    assert abs(kept - (1 - q)) <= 6 * (q * (1 - q) / n) ** 0.5
    assert abs(a.double().mean().item() - 1) <= 6 * (q / (1 - q) / n) ** 0.5
    for b in (ue.dropout_forward(x, p, 2, 0), ue.dropout_forward(x, p, 1, 1), ue.dropout_forward(x, p, 1 + (1 << 32), 0)):
        both = ((a == 0) & (b == 0)).double().mean().item()
        assert abs(both - q * q) <= 6 * (q * q * (1 - q * q) / n) ** 0.5


def test_gradient():
    """The gradient is the mask's own: exact, and equal to differences (dropout
    is linear, so a difference of any step is the gradient)."""
    x = torch.randn(37, 65, device="cuda", requires_grad=True)
    r = torch.randn(37, 65, device="cuda", requires_grad=True)
    dy = torch.randn(37, 65, device="cuda")
    y = dropout(x, 0.3, 11, 4, residual=r)
    dx, dr = torch.autograd.grad(y, (x, r), dy)
    assert torch.equal(dr, dy) and torch.equal(dx.cpu(), expected(dy, 0.3, 11, 4))
    step = torch.zeros_like(x)
    step[5, 6] = step[20, 64] = 1.0
    fd = ue.dropout_forward(x.detach() + step, 0.3, 11, 4).double() - ue.dropout_forward(x.detach(), 0.3, 11, 4).double()
    got = dx.double() * step.double() / torch.where(dy == 0, 1.0, dy.double())
    # a survivor's difference carries the rounding of values below 8, twice
    assert torch.allclose(fd, got, atol=2 * 8 * 2.0 ** -23, rtol=0)


def test_in_place_views_and_module():
    x = torch.randn(1001, device="cuda").to(torch.bfloat16)
    want = ue.dropout_forward(x, 0.2, 5, 6, residual=x)
    v = torch.zeros(1002, device="cuda", dtype=torch.bfloat16)
    v[1:] = x
    assert torch.equal(ue.dropout_forward(v[1:], 0.2, 5, 6, residual=x), want)      # starts at an odd element
    assert ue.dropout_forward(v[1:], 0.2, 5, 6, residual=v[1:], out=v[1:]).data_ptr() == v[1:].data_ptr()
    assert torch.equal(v[1:], want) and v[0] == 0
    assert ue.dropout_forward(x[:0], 0.2, 5).numel() == 0
    m = Dropout(0.2, seed=9, layer_id=2)
    a, b = m(x), m(x)
    assert torch.equal(a, ue.dropout_forward(x, 0.2, 9, 2)) and torch.equal(b, ue.dropout_forward(x, 0.2, 10, 2))
    m.eval()
    assert m(x) is x


def test_counters_past_32_bits():
    n = 2 ** 31 + 4096 + 3
    say("dropout large", n)
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    y = ue.dropout_forward(x, 0.25, 77, 8)
    for first in (0, 2 ** 31 - 64, 2 ** 31 + 8, n - 1000):
        k = min(1000, n - first)
        assert torch.equal(y[first:first + k].cpu(), expected(x[first:first + k], 0.25, 77, 8, first=first))
