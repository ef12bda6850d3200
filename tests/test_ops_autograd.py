"""Forward-mode differentiation through the operators around the linear
layers: refused, with and without a gradient asked for, as they have no
tangents (on the host: the refusal comes before any check of the device)."""

import pytest
import torch
from torch.autograd import forward_ad

from paper_2609_02846_amd.dropout import Dropout, dropout
from paper_2609_02846_amd.fp8 import Fp8Linear, fp8_linear
from paper_2609_02846_amd.norm import LayerNorm, layer_norm
from paper_2609_02846_amd.sublayer import PreNormSublayer, sublayer


def bf16(*shape):
    return torch.randn(*shape).to(torch.bfloat16)


def frozen():
    layer = Fp8Linear(8, 8, device="cpu")
    layer.frozen = (layer.weight.detach(), torch.ones(1))
    return layer


W, V = bf16(8, 8), bf16(8)
CALLS = {
    "layer_norm": lambda x: layer_norm(x, V, V),
    "layer_norm module": lambda x: LayerNorm(8, device="cpu")(x),
    "layer_norm weight": lambda x: layer_norm(W, x[0], V),
    "layer_norm bias": lambda x: layer_norm(W, None, x[0]),
    "dropout": lambda x: dropout(x, 0.1, 1),
    "dropout residual": lambda x: dropout(W, 0.1, 1, residual=x),
    "dropout module": lambda x: Dropout(0.1)(x),
    "fp8_linear": lambda x: fp8_linear(x, W),
    "fp8_linear weight": lambda x: fp8_linear(W, x),
    "frozen": lambda x: frozen()(x),
    "sublayer": lambda x: sublayer(x, V, V, W),
    "sublayer gain": lambda x: sublayer(W, x[0], None, W),
    "sublayer weight": lambda x: sublayer(W, V, V, x),
    "sublayer module": lambda x: PreNormSublayer(8, device="cpu")(x),
}


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("what", CALLS)
def test_tangents_are_refused(what, grad):
    with forward_ad.dual_level(), torch.set_grad_enabled(grad):
        x = forward_ad.make_dual(bf16(8, 8), bf16(8, 8))
        with pytest.raises(NotImplementedError, match="forward-mode"):
            CALLS[what](x)


def test_plain_tensors_inside_a_dual_level_are_not():
    with forward_ad.dual_level():
        for call in CALLS.values():
            with pytest.raises(ValueError):           # host tensors, nothing else
                call(bf16(8, 8))
