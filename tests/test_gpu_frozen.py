"""Frozen 8-bit layers and branches on the GPU, where gradients are recorded
and where the weight changes."""

import pytest
import torch

from paper_2609_02846_amd.fp8 import Fp8Linear
from paper_2609_02846_amd.sublayer import PreNormSublayer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("training", [True, False])
def test_frozen_branch(training):
    m = PreNormSublayer(256, p=0.0).train(training)
    x = torch.randn(20, 256, device="cuda").to(torch.bfloat16)
    with torch.no_grad():
        m.linear.freeze()
        want = m(x)
    y = m(x.requires_grad_())
    assert torch.equal(y, want)
    with pytest.raises(RuntimeError, match="unfreeze"):
        y.float().sum().backward()
    m.linear.unfreeze()
    m(x).float().sum().backward()
    assert x.grad is not None and all(p.grad is not None for p in m.parameters())


def test_loading_into_a_frozen_layer():
    x = torch.randn(5, 300, device="cuda").to(torch.bfloat16)
    layer, other = Fp8Linear(300, 200).freeze(), Fp8Linear(300, 200)
    with torch.no_grad():
        before = layer(x)
        layer.load_state_dict(other.state_dict())
        assert torch.equal(layer(x), other(x)) and not torch.equal(layer(x), before)
