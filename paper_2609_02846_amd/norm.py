"""Layer norm as an autograd function and a module, on the library's kernels."""

import torch
from torch.autograd.function import once_differentiable

from . import _check, _stream, load_library
from .operators import _TYPES, _like, layer_norm_forward, norm_args, recorded

# Small calls are bound by the host: the autograd function marshals the library
# calls itself, and both statistics of a row lie in one buffer.


class _LayerNormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        pt, rows, C = norm_args(x, weight, bias)
        xt = _TYPES[x.dtype]
        y, stats = torch.empty_like(x), torch.empty(2 * rows, dtype=torch.float32, device=x.device)
        mean = stats.data_ptr()
        _check(load_library().ue5m3_layer_norm(x.data_ptr(), rows, C, xt, None if weight is None else weight.data_ptr(),
                                               None if bias is None else bias.data_ptr(), pt, eps, y.data_ptr(), mean,
                                               mean + 4 * rows, _stream()), "ue5m3_layer_norm")
        ctx.save_for_backward(x, weight, stats)
        ctx.args = rows, C, xt, pt, x.dtype if pt == xt else torch.float32
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, stats = ctx.saved_tensors
        rows, C, xt, pt, pdtype = ctx.args
        need_x, need_w, need_b, _ = ctx.needs_input_grad
        dy = _like(dy.contiguous(), x, "the output gradient")
        dx = torch.empty_like(x) if need_x else None
        dw = torch.empty(C, dtype=pdtype, device=x.device) if need_w else None
        db = torch.empty(C, dtype=pdtype, device=x.device) if need_b else None
        mean = stats.data_ptr()
        _check(load_library().ue5m3_layer_norm_grad(
            x.data_ptr(), dy.data_ptr(), rows, C, xt, None if weight is None else weight.data_ptr(), pt, mean,
            mean + 4 * rows, None, dx.data_ptr() if need_x else None, dw.data_ptr() if need_w else None,
            db.data_ptr() if need_b else None, _stream()), "ue5m3_layer_norm_grad")
        return dx, dw, db, None


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over the last dimension of ``x`` (bf16, fp16 or fp32), with
    gradients.  ``weight`` and ``bias`` have x's type or fp32; their gradients
    are summed in fp32 in a fixed order."""
    x = x.contiguous()
    if recorded(x, weight, bias):
        return _LayerNormFn.apply(x, weight, bias, float(eps))
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
