"""Layer norm as an autograd function and a module, on the library's kernels."""

import torch
from torch.autograd.function import once_differentiable

from .operators import layer_norm_forward, layer_norm_grad


class _LayerNormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = layer_norm_forward(x, weight, bias, eps, stats=True)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.param_dtype = None if bias is None else bias.dtype
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        dx, dw, db = layer_norm_grad(x, dy.contiguous(), weight, mean, rstd, need=ctx.needs_input_grad[:3],
                                     param_dtype=ctx.param_dtype)
        return dx, dw, db, None


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over the last dimension of ``x`` (bf16, fp16 or fp32), with
    gradients.  ``weight`` and ``bias`` have x's type or fp32; their gradients
    are summed in fp32 in a fixed order."""
    x = x.contiguous()
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, weight, bias)):
        return _LayerNormFn.apply(x, weight, bias, eps)
    return layer_norm_forward(x, weight, bias, eps)


class LayerNorm(torch.nn.Module):
    """Layer norm over a last dimension of ``features``."""

    def __init__(self, features, eps=1e-5, bias=True, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.features, self.eps = int(features), float(eps)
        self.weight = torch.nn.Parameter(torch.ones(self.features, dtype=dtype, device=device))
        self.bias = torch.nn.Parameter(torch.zeros(self.features, dtype=dtype, device=device)) if bias else None

    def forward(self, x):
        return layer_norm(x, self.weight, self.bias, self.eps)

    def extra_repr(self):
        return f"{self.features}, eps={self.eps}"
