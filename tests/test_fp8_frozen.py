"""A frozen 8-bit layer on the host, with a stand-in for its kernels: what it
does where gradients are asked for."""

import pytest
import torch

from paper_2609_02846_amd import fp8
from paper_2609_02846_amd.fp8 import Fp8Linear
from paper_2609_02846_amd.sublayer import PreNormSublayer


@pytest.fixture(autouse=True)
def stand_in(monkeypatch):
    monkeypatch.setattr(fp8, "quantize_fp8_tiles", lambda w, scale, transposed: (w.clone(), torch.ones(1), None, None))
    monkeypatch.setattr(fp8, "linear_fp8", lambda x, w, s: x @ w.t())
    monkeypatch.setattr("paper_2609_02846_amd.norm.layer_norm",
                        lambda x, w, b, eps: torch.nn.functional.layer_norm(x, w.shape, w, b, eps))
    monkeypatch.setattr("paper_2609_02846_amd.dropout.dropout_forward",
                        lambda x, p, seed, tensor_id, residual=None: x if residual is None else x + residual)


def branch():
    return PreNormSublayer(16, device="cpu")


def test_a_backward_pass_through_a_frozen_layer_raises():
    """Its forward result stands; gradients past it would be missing terms."""
    x = torch.randn(3, 16).to(torch.bfloat16)
    layer = Fp8Linear(16, 8, device="cpu")
    plain = layer.freeze()(x)
    assert not plain.requires_grad
    y = layer(x.requires_grad_())
    assert torch.equal(y, plain)
    with pytest.raises(RuntimeError, match="unfreeze"):
        y.sum().backward()


@pytest.mark.parametrize("training", [True, False])
def test_a_frozen_branch_gives_no_partial_gradients(training):
    m = branch().train(training)
    m.linear.freeze()
    x = torch.randn(3, 16).to(torch.bfloat16).requires_grad_()
    y = m(x)
    with pytest.raises(RuntimeError, match="unfreeze"):
        y.sum().backward()
    with torch.no_grad():
        assert not m(x).requires_grad


def test_a_loaded_weight_is_quantized_again():
    """A frozen layer answers with the weight that it holds, not with the one
    that it was frozen with."""
    x = torch.randn(3, 16).to(torch.bfloat16)
    layer, other = Fp8Linear(16, 8, device="cpu").freeze(), Fp8Linear(16, 8, device="cpu")
    stack = torch.nn.Sequential(layer)
    with torch.no_grad():
        stack.load_state_dict({"0.weight": other.weight.clone()})
        assert torch.equal(stack(x), other.freeze()(x))
    assert layer.frozen is not None


def test_a_moved_layer_stays_whole():
    """.to() takes the quantized weight along."""
    layer = Fp8Linear(16, 8, device="cpu").freeze()
    layer.to("meta")
    assert all(t.device.type == "meta" for t in (layer.weight, *layer.frozen))
