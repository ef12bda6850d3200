"""The residual branch and dropout under activation checkpointing: the results
and gradients of the same calls without it."""

import pytest
import torch
from torch.utils.checkpoint import checkpoint

from paper_2609_02846_amd.dropout import Dropout
from paper_2609_02846_amd.sublayer import PreNormSublayer

pytestmark = pytest.mark.gpu


def outcome(modules, x, reentrant=None):
    """Result and gradients of the modules in a chain, two turns of it."""
    torch.manual_seed(11)
    x = x.clone().requires_grad_()
    params = [p for m in modules for p in m.parameters()]
    y = x
    for m in modules * 2:
        y = m(y) if reentrant is None else checkpoint(m, y, use_reentrant=reentrant)
    leaves = [x] + params
    for t in leaves:
        t.grad = None
    y.float().square().sum().backward()              # (autograd.grad does not go through reentrant checkpoints)
    return [y.detach()] + [t.grad for t in leaves]


@pytest.mark.parametrize("reentrant", [True, False])
def test_branch(reentrant):
    modules = [PreNormSublayer(256, p=0.2), PreNormSublayer(256, p=0.3, scale="f32")]
    x = torch.randn(40, 256, device="cuda").to(torch.bfloat16)
    for got, want in zip(outcome(modules, x, reentrant), outcome(modules, x)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("reentrant", [True, False])
def test_dropout(reentrant):
    modules = [Dropout(0.2), Dropout(0.2)]
    x = torch.randn(33, 77, device="cuda")
    for got, want in zip(outcome(modules, x, reentrant), outcome(modules, x)):
        assert torch.equal(got, want)


def test_a_stack_has_a_mask_for_each_layer():
    x = torch.ones(64, 256, device="cuda", dtype=torch.bfloat16)
    a, b = Dropout(0.5), Dropout(0.5)
    assert not torch.equal(a(x), b(x)) and not torch.equal(a(x), a(x))


@pytest.mark.parametrize("reentrant", [True, False])
def test_counted_keys_are_refused(reentrant):
    x = torch.randn(8, 128, device="cuda").to(torch.bfloat16)
    with pytest.raises(RuntimeError, match="seed"):
        outcome([PreNormSublayer(128, seed=4)], x, reentrant)
