"""A pre-norm residual branch, x + dropout(linear(layer_norm(x))), in training:
layer norm, the 8-bit linear layer and dropout together.

One autograd function, so that what the branch's ends share is joined: the
residual is added in dropout's pass, and its gradient in the norm's backward
pass.  Between the operators bf16 tensors are handed on, as between the
separate calls, and the results are theirs.
"""

import torch
from torch.autograd.function import once_differentiable

from .dropout import Dropout
from .fp8 import Fp8Linear, _check_formats, _flat, backward_products, forward_product
from .norm import LayerNorm
from .operators import dropout_forward, layer_norm_forward, layer_norm_grad


class _SublayerFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gain, bias, w, p, seed, tensor_id, eps, scale, grad_fmt, need_w):
        h, mean, rstd = layer_norm_forward(x, gain, bias, eps, stats=True)
        y, keep = forward_product(h, w, scale, True, need_w)
        ctx.save_for_backward(x, gain, mean, rstd, keep)
        ctx.args = (*x.shape, w.shape[0], scale, grad_fmt, True, need_w)
        ctx.key, ctx.param_dtype = (p, seed, tensor_id), None if bias is None else bias.dtype
        return dropout_forward(y, p, seed, tensor_id, residual=x, out=y)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        x, gain, mean, rstd, keep = ctx.saved_tensors
        dout = dout.to(torch.bfloat16).contiguous()
        dh, dw = backward_products(dropout_forward(dout, *ctx.key), keep, *ctx.args)
        dx, dgain, dbias = layer_norm_grad(x, dh, gain, mean, rstd, residual_grad=dout,
                                           need=ctx.needs_input_grad[:3], param_dtype=ctx.param_dtype)
        return dx, dgain, dbias, dw, None, None, None, None, None, None, None


def sublayer(x, gain, bias, weight, p=0.1, seed=0, tensor_id=0, eps=1e-5, scale="e8m0", grad_fmt="e4m3"):
    """x + dropout(fp8_linear(layer_norm(x, gain, bias), weight)) for bf16
    ``x`` [..., C] and ``weight`` [C, C], with gradients."""
    _check_formats(scale, grad_fmt)
    C = x.shape[-1]
    if tuple(weight.shape) != (C, C):
        raise ValueError(f"the branch's weight must be [{C}, {C}] to add to its input")
    x2 = _flat(x, C)
    grad = torch.is_grad_enabled()
    if grad and any(t is not None and t.requires_grad for t in (x, gain, bias, weight)):
        y = _SublayerFn.apply(x2, gain, bias, weight, float(p), int(seed), int(tensor_id), float(eps), scale, grad_fmt,
                              weight.requires_grad)
    else:
        h = layer_norm_forward(x2, gain, bias, eps)
        y, _ = forward_product(h, weight, scale, False, False)
        y = dropout_forward(y, p, seed, tensor_id, residual=x2, out=y)
    return y.reshape(x.shape)


class PreNormSublayer(torch.nn.Module):
    """The branch with its parameters.  In evaluation dropout passes and, after
    ``linear.freeze()``, the product takes the quantized weight."""

    def __init__(self, features, p=0.1, eps=1e-5, scale="e8m0", grad_fmt="e4m3", seed=0, layer_id=0, device="cuda"):
        super().__init__()
        self.norm = LayerNorm(features, eps, device=device)
        self.linear = Fp8Linear(features, features, scale, grad_fmt, device)
        self.dropout = Dropout(p, seed, layer_id)

    def forward(self, x):
        if not self.training or self.linear.frozen is not None:
            return self.dropout(self.linear(self.norm(x)), residual=x)
        d = self.dropout
        key = (d.seed + d.calls) & (2 ** 64 - 1)
        d.calls += 1
        return sublayer(x, self.norm.weight, self.norm.bias, self.linear.weight, d.p, key, d.layer_id, self.norm.eps,
                        self.linear.scale, self.linear.grad_fmt)
