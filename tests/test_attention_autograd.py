"""Rotation, attention, the paged cache and the attention branch under autograd, on
the host (the refusals come before any check of the device): forward-mode
tangents, gradients that a call would drop, casts of the branch."""

import pytest
import torch
from torch.autograd import forward_ad

from paper_2609_02846_amd import AttentionC, AttentionGradC, load_library
from paper_2609_02846_amd.attention import attention, paged_attention
from paper_2609_02846_amd.paged import copy_pages
from paper_2609_02846_amd.rotary import qk_norm_rope, qk_norm_rope_append
from paper_2609_02846_amd.sublayer import PreNormAttention


def heads():
    return torch.randn(4, 2, 32).to(torch.bfloat16)


H, F, W = heads(), torch.ones(16), torch.ones(32)
C, N = torch.zeros(3, 16, 2, 32, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
SERVING = {
    "append q": lambda x: qk_norm_rope_append(x, H, H, C, C, N, freqs=F),
    "append v": lambda x: qk_norm_rope_append(H, H, x, C, C, N, freqs=F),
    "append weight": lambda x: qk_norm_rope_append(H, H, H, C, C, N, k_weight=x[0, 0], freqs=F),
    "append frequencies": lambda x: qk_norm_rope_append(H, H, H, C, C, N, freqs=x[0, 0, :16].float()),
    "append cache": lambda x: qk_norm_rope_append(H, H, H, x[None], C, N, freqs=F),
    "paged q": lambda x: paged_attention(x, C, C, N[None].int(), N.int()),
    "paged cache": lambda x: paged_attention(H, C, x[None], N[None].int(), N.int()),
    "copy": lambda x: copy_pages(x, [0], [1]),
}
CALLS = {
    "rope q": lambda x: qk_norm_rope(x, H, freqs=F),
    "rope k": lambda x: qk_norm_rope(H, x, freqs=F),
    "rope weight": lambda x: qk_norm_rope(H, H, W, x[0, 0].float(), freqs=F),
    "rope frequencies": lambda x: qk_norm_rope(H, H, freqs=x[0, 0, :16].float()),
    "attention q": lambda x: attention(x, H, H),
    "attention k": lambda x: attention(H, x, H),
    "attention v": lambda x: attention(H, H, x),
    "branch": lambda x: PreNormAttention(32, 2, 1, 16, device="cpu")(x),
    **SERVING,
}


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("what", CALLS)
def test_tangents_are_refused(what, grad):
    with forward_ad.dual_level(), torch.set_grad_enabled(grad):
        x = forward_ad.make_dual(heads(), heads())
        with pytest.raises(NotImplementedError, match="forward-mode"):
            CALLS[what](x)


@pytest.mark.parametrize("what", SERVING)
def test_serving_calls_drop_no_gradient(what):
    x = heads().requires_grad_()
    with pytest.raises(RuntimeError, match="no gradients"):
        SERVING[what](x)
    with torch.no_grad(), pytest.raises(ValueError):  # host tensors
        SERVING[what](x)


def test_frequencies_have_no_gradient():
    with pytest.raises((ValueError, RuntimeError)):
        qk_norm_rope(H, H, freqs=F.clone().requires_grad_())


def test_gradients_are_of_bf16():
    """The library's own entry refuses fp16 as the binding does, before any pointer."""
    lib = load_library()
    sizes = dict(q_tokens=0, k_tokens=0, sequences=1, q_heads=4, kv_heads=2, dim=64, causal=1, scale=0.1, q_token=256, q_head=64,
                 k_token=128, k_head=64, v_token=128, v_head=64)
    assert lib.ue5m3_attention_grad(AttentionC(type=0, **sizes), AttentionGradC(), None) == 0
    assert lib.ue5m3_attention_grad(AttentionC(type=1, **sizes), AttentionGradC(), None) == 1
    assert lib.ue5m3_attention(AttentionC(type=1, **sizes), None, None) == 0


def test_the_branch_keeps_its_frequencies():
    """Sixteen bits of them would be off by turns at far positions."""
    m = PreNormAttention(64, 2, 1, 32, device="cpu")
    freqs = m.freqs.clone()
    for cast in (lambda: m.bfloat16(), lambda: m.to("cpu", torch.bfloat16), lambda: m.to("cpu")):
        cast()
        assert m.freqs.dtype == torch.float32 and torch.equal(m.freqs, freqs)
    assert "freqs" not in m.state_dict()
