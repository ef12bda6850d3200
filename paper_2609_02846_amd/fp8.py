"""A linear layer in 8-bit floating point with one scale for each block of 128:
for layers that stay out of FP4.

Y = X W^T, dX = dY W and dW = dY^T X on operands quantized in blocks of 128
along each product's own contraction: X and dY along their rows and down their
columns (both from one read), W in 128 x 128 tiles whose values the forward and
the input gradient's product share.  X and W are E4M3, dY is E4M3 or E5M2
(wider range).  Scales come from the blocks themselves, so there is no state.
The outputs are bf16; the products' own arithmetic (see ue5m3_gemm_fp8) is 4e-5
to 7e-5 from the exact sums in relative L2 norm, 1 / 24 of bf16's rounding.
"""

import functools

import torch
from torch.autograd.function import once_differentiable

from . import NN, NT, OUT_BF16, TN, _bf16_2d, _check, _numel, _stream, load_library
from .linear import _Layout
from .operators import COL128T, ROW128, TILE128, linear_fp8, pad128, quantize_fp8_tiles, recorded, scale_pitch

_GRAD = {"e4m3": 0, "e5m2": 1}
_SCALE = {"f32": (0, 4), "e8m0": (1, 1)}             # code, bytes of a scale


@functools.lru_cache(maxsize=512)
def _forward_layout(T, K, N, size, need_dx, need_dw):
    """(saved, temp): operands that the backward pass reads (X down its columns
    for dW, the transposed weight for dX), and those that only Y needs."""
    saved, temp = _Layout(), _Layout()
    kb, nb, tb = pad128(K) // 128, pad128(N) // 128, pad128(T) // 128
    temp.x, temp.sx = temp.add(T * kb * 128), temp.add(kb * scale_pitch(T) * size)
    temp.w, temp.sw = temp.add(N * kb * 128), temp.add(kb * nb * size)
    if need_dw:
        saved.xt, saved.sxt = saved.add(K * tb * 128), saved.add(tb * scale_pitch(K) * size)
    if need_dx:
        saved.wt, saved.swt = saved.add(K * nb * 128), saved.add(kb * nb * size)
    return saved, temp


@functools.lru_cache(maxsize=512)
def _backward_layout(T, N, size, need_dx, need_dw):
    temp = _Layout()
    nb, tb = pad128(N) // 128, pad128(T) // 128
    if need_dx:
        temp.d, temp.sd = temp.add(T * nb * 128), temp.add(nb * scale_pitch(T) * size)
    if need_dw:
        temp.dt, temp.sdt = temp.add(N * tb * 128), temp.add(tb * scale_pitch(N) * size)
    return temp


def _buffer(layout, like):
    return torch.empty(layout.bytes, dtype=torch.uint8, device=like.device)


def forward_product(x, w, scale, need_dx, need_dw):
    """Y of 2-D bf16 ``x`` and ``w``, and the buffer of operands that
    ``backward_products`` takes."""
    _bf16_2d(x, "x")
    _bf16_2d(w, "weight")
    T, K = x.shape
    N = w.shape[0]
    if w.shape[1] != K or w.device != x.device:
        raise ValueError(f"weight has {w.shape[1]} columns on {w.device}, the input {K} on {x.device}")
    kind, size = _SCALE[scale]
    lib, stream = load_library(), _stream()
    saved, temp = _forward_layout(T, K, N, size, need_dx, need_dw)
    work, y = _buffer(temp, x), torch.empty((T, N), dtype=torch.bfloat16, device=x.device)
    keep = _buffer(saved, x) if need_dx or need_dw else None
    t, k = work.data_ptr(), keep.data_ptr() if keep is not None else 0
    xt, sxt = (k + saved.xt, k + saved.sxt) if need_dw else (None, None)
    wt, swt = (k + saved.wt, k + saved.swt) if need_dx else (None, None)
    _check(lib.ue5m3_quantize_fp8(x.data_ptr(), T, K, 0, 0, kind, t + temp.x, t + temp.sx, xt, sxt, stream),
           "ue5m3_quantize_fp8")
    _check(lib.ue5m3_quantize_fp8_tiles(w.data_ptr(), N, K, 0, kind, t + temp.w, t + temp.sw, wt, swt, stream),
           "ue5m3_quantize_fp8_tiles")
    _check(lib.ue5m3_gemm_fp8(NT, T, N, K, t + temp.x, t + temp.sx, ROW128, 0, t + temp.w, t + temp.sw, TILE128, kind,
                              y.data_ptr(), OUT_BF16, stream), "ue5m3_gemm_fp8")
    return y, keep


def backward_products(dy, keep, T, K, N, scale, grad_fmt, need_dx, need_dw):
    """(dX, dW) in bf16 for the output gradient ``dy`` [T, N]; ``keep`` from
    ``forward_product`` with the same needs."""
    _bf16_2d(dy, "the output gradient")
    kind, size = _SCALE[scale]
    fmt, lib, stream = _GRAD[grad_fmt], load_library(), _stream()
    saved, _ = _forward_layout(T, K, N, size, need_dx, need_dw)
    temp = _backward_layout(T, N, size, need_dx, need_dw)
    work = _buffer(temp, dy)
    t, k = work.data_ptr(), keep.data_ptr()
    dx = dw = None
    d, sd = (t + temp.d, t + temp.sd) if need_dx else (None, None)
    dt, sdt = (t + temp.dt, t + temp.sdt) if need_dw else (None, None)
    _check(lib.ue5m3_quantize_fp8(dy.data_ptr(), T, N, 0, fmt, kind, d, sd, dt, sdt, stream), "ue5m3_quantize_fp8")
    if need_dx:
        dx = torch.empty((T, K), dtype=torch.bfloat16, device=dy.device)
        _check(lib.ue5m3_gemm_fp8(NN, T, K, N, d, sd, ROW128, fmt, k + saved.wt, k + saved.swt, TILE128, kind,
                                  dx.data_ptr(), OUT_BF16, stream), "ue5m3_gemm_fp8")
    if need_dw:
        dw = torch.empty((N, K), dtype=torch.bfloat16, device=dy.device)
        _check(lib.ue5m3_gemm_fp8(TN, N, K, T, dt, sdt, COL128T, fmt, k + saved.xt, k + saved.sxt, COL128T, kind,
                                  dw.data_ptr(), OUT_BF16, stream), "ue5m3_gemm_fp8")
    return dx, dw


class _Fp8LinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, scale, grad_fmt, need_dx, need_dw):
        y, keep = forward_product(x, w, scale, need_dx, need_dw)
        ctx.args = (*x.shape, w.shape[0], scale, grad_fmt, need_dx, need_dw)
        ctx.save_for_backward(keep)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        keep, = ctx.saved_tensors
        dx, dw = backward_products(dy.to(torch.bfloat16).contiguous(), keep, *ctx.args)
        return dx, dw, None, None, None, None


def _check_formats(scale, grad_fmt):
    if scale not in _SCALE:
        raise ValueError(f"scale must be one of {sorted(_SCALE)}")
    if grad_fmt not in _GRAD:
        raise ValueError(f"grad_fmt must be one of {sorted(_GRAD)}")


def _flat(x, features):
    if x.dtype != torch.bfloat16 or x.dim() == 0 or x.shape[-1] != features:
        raise ValueError(f"input must be bf16 with last dimension {features}")
    return x.contiguous() if x.dim() == 2 else x.reshape(_numel(x.shape[:-1]), features).contiguous()


def fp8_linear(x, weight, scale="e8m0", grad_fmt="e4m3"):
    """``x`` [..., K] times ``weight`` [N, K] transposed (both bf16), with
    gradients; every size is allowed.  ``scale``: "e8m0" (powers of two, the
    matrix instructions' own) or "f32"; ``grad_fmt``: format of the output
    gradient, "e4m3" or "e5m2"."""
    _check_formats(scale, grad_fmt)
    x2 = _flat(x, weight.shape[1])
    if recorded(x2, weight):
        need_dx, need_dw = x.requires_grad, weight.requires_grad
        y = _Fp8LinearFn.apply(x2, weight, scale, grad_fmt, need_dx, need_dw)
    else:
        y, _ = forward_product(x2, weight, scale, False, False)
    return y if x.dim() == 2 else y.reshape(*x.shape[:-1], weight.shape[0])


class _FrozenFn(torch.autograd.Function):
    """The serving call where gradients are recorded: in a sum with another
    branch they would reach that one alone, without a word."""

    @staticmethod
    def forward(ctx, x, w, scales):
        return linear_fp8(x.contiguous(), w, scales)

    @staticmethod
    def backward(ctx, dy):
        raise RuntimeError("a frozen Fp8Linear has no gradients: unfreeze() it, or call it under torch.no_grad()")


class Fp8Linear(torch.nn.Module):
    """Linear layer without bias in 8-bit floating point (see ``fp8_linear``).
    ``freeze()`` quantizes the weight once for serving: forward calls then take
    the quantized weight, and a backward pass through one raises, until
    ``unfreeze()``.  A weight changed in place while frozen (an optimizer's
    step) needs another ``freeze()``."""

    def __init__(self, in_features, out_features, scale="e8m0", grad_fmt="e4m3", device="cuda"):
        super().__init__()
        _check_formats(scale, grad_fmt)
        self.in_features, self.out_features = int(in_features), int(out_features)
        self.scale, self.grad_fmt, self.frozen = scale, grad_fmt, None
        self.weight = torch.nn.Parameter(torch.empty(out_features, in_features, dtype=torch.bfloat16, device=device))
        torch.nn.init.normal_(self.weight, std=in_features ** -0.5)

    def freeze(self):
        self.frozen = quantize_fp8_tiles(self.weight.detach(), self.scale, transposed=False)[:2]
        return self

    def unfreeze(self):
        self.frozen = None
        return self

    # What was quantized goes with the weight: a loaded one is quantized in its
    # place, a moved one takes it along.
    def _load_from_state_dict(self, *args):
        super()._load_from_state_dict(*args)
        if self.frozen is not None:
            self.freeze()

    def _apply(self, fn, recurse=True):
        super()._apply(fn, recurse)
        if self.frozen is not None:
            self.frozen = tuple(t.to(self.weight.device) for t in self.frozen)
        return self

    def forward(self, x):
        if self.frozen is None:
            return fp8_linear(x, self.weight, self.scale, self.grad_fmt)
        if recorded(x):
            return _FrozenFn.apply(x, *self.frozen)
        return linear_fp8(x.contiguous(), *self.frozen)

    def extra_repr(self):
        return f"in_features={self.in_features}, out_features={self.out_features}, scale={self.scale}"
