"""Binding of the operators around the linear layers: layer norm, dropout, and
a linear layer's products in 8-bit floating point with one scale for each block
of 128.  As in the rest of the binding, every step runs in the library's HIP
kernels; this module checks and marshals arguments.

8-bit tensors are ``torch.float8_e4m3fn`` or ``torch.float8_e5m2``; block
scales are fp32, or uint8 E8M0 codes (powers of two, which the matrix
instructions apply themselves).  A quantized [R, C] tensor is

  row blocks      payload [R, pad(C)], scales [pad(C) / 128, pitch(R)]
  column blocks   payload [C, pad(R)], scales [pad(R) / 128, pitch(C)]
                  (stored transposed)
  tiles           payload [R, pad(C)], scales [pad(R) / 128, pad(C) / 128],
                  and the transposed copy of both

with pad() up to a multiple of 128 and pitch() up to one of 16.
"""

import contextlib

import torch
from torch.autograd import forward_ad

from . import _LAYOUTS, NT, OUT_BF16, OUT_F32, TN, _check, _dev_buf, _numel, _ptr, _stream, load_library

BF16, F16, F32 = range(3)
_TYPES = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_FP8_CODES = {torch.float8_e4m3fn: 0, torch.float8_e5m2: 1}
SCALE = {"f32": torch.float32, "e8m0": torch.uint8}
_SCALE_CODES = {torch.float32: 0, torch.uint8: 1}
ROW128, COL128T, TILE128 = 6, 7, 8
_BLOCKINGS = {"row": ROW128, "colT": COL128T, "tile": TILE128}


def pad128(n):
    return (n + 127) // 128 * 128


def scale_pitch(n):
    return (n + 15) // 16 * 16


def _on(stream):
    """Outputs of a call on ``stream`` are that stream's memory, as torch's
    allocator counts it."""
    return _HERE if stream is None else torch.cuda.stream(stream)


_HERE = contextlib.nullcontext()


def _tensor(t, name, dtypes, like=None, dim=None):
    """A dense device tensor of one of ``dtypes``, on the current device or
    that of ``like``."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in dtypes or not t.is_contiguous():
        names = ", ".join(str(d) for d in dtypes)
        raise ValueError(f"{name} must be a contiguous CUDA/HIP tensor of {names}")
    if dim is not None and t.dim() != dim:
        raise ValueError(f"{name} must have {dim} dimensions, not {t.dim()}")
    if t.get_device() != (torch._C._cuda_getDevice() if like is None else like.get_device()):
        raise ValueError(f"{name} is on {t.device}, not on the device of the call")
    return t


def _like(t, x, name):
    """``t`` (or None) with the shape, type and device of ``x``."""
    if t is not None and _tensor(t, name, (x.dtype,), x).shape != x.shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, {tuple(x.shape)} needed")
    return t


def recorded(*tensors):
    """Whether autograd records a call on these tensors (or None).  Tangents of
    forward-mode differentiation are refused: no operator here has any, and
    where nothing is recorded they would be dropped."""
    if forward_ad._current_level >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None
                                              for t in tensors):
        raise NotImplementedError("the operators have no forward-mode derivatives")
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


# ------------------------------------------------------------- layer norm --
def _affine(x, weight, bias):
    """Element type code of the parameters."""
    C, dtype = x.shape[-1], None
    for t, name in ((weight, "weight"), (bias, "bias")):
        if t is None:
            continue
        _tensor(t, name, (x.dtype, torch.float32), x)
        if t.numel() != C or t.dim() != 1:
            raise ValueError(f"{name} must have one dimension of {C}")
        if dtype is not None and t.dtype != dtype:
            raise ValueError("weight and bias must have one type")
        dtype = t.dtype
    return _TYPES[x.dtype if dtype is None else dtype]


def norm_args(x, weight, bias):
    """Checks; element type code of the parameters, rows and columns."""
    _tensor(x, "x", _TYPES)
    if x.dim() == 0:
        raise ValueError("x must have a dimension to normalise")
    C = x.shape[-1]
    return _affine(x, weight, bias), x.numel() // C if C else 0, C


def layer_norm_forward(x, weight=None, bias=None, eps=1e-5, stats=False, out=None, stream=None):
    """Layer norm over the last dimension of ``x`` (bf16, fp16 or fp32; see
    ue5m3_layer_norm).  ``weight`` and ``bias``: of x's type or fp32, or None.
    Returns y, with ``stats`` (y, mean, rstd): the fp32 statistics of the rows,
    which ``layer_norm_grad`` takes."""
    pt, rows, C = norm_args(x, weight, bias)
    with _on(stream):
        y = torch.empty_like(x) if out is None else _like(out, x, "out")
        mean, rstd = torch.empty((2, rows), dtype=torch.float32, device=x.device) if stats else (None, None)
    _check(load_library().ue5m3_layer_norm(_ptr(x), rows, C, _TYPES[x.dtype], _ptr(weight), _ptr(bias), pt, float(eps),
                                           _ptr(y), _ptr(mean), _ptr(rstd), _stream(stream)), "ue5m3_layer_norm")
    return (y, mean, rstd) if stats else y


def layer_norm_grad(x, dy, weight, mean, rstd, residual_grad=None, need=(True, True, True), param_dtype=None,
                    stream=None):
    """Gradients of ``layer_norm_forward`` (see ue5m3_layer_norm_grad): (dx,
    dweight, dbias), each None where ``need`` says so.  ``residual_grad`` is
    added to dx.  dweight and dbias have the type of ``weight``, or
    ``param_dtype`` where that is None."""
    _tensor(x, "x", _TYPES)
    _like(dy, x, "dy")
    _like(residual_grad, x, "residual_grad")
    pt, C = _affine(x, weight, None), x.shape[-1]
    if weight is None and param_dtype is not None:
        if param_dtype not in (x.dtype, torch.float32):
            raise ValueError("the parameters have x's type or fp32")
        pt = _TYPES[param_dtype]
    rows = x.numel() // C if C else 0
    for t, name in ((mean, "mean"), (rstd, "rstd")):
        _dev_buf(t, torch.float32, rows, name)
    pdtype = (x.dtype if param_dtype is None else param_dtype) if weight is None else weight.dtype
    with _on(stream):
        dx = torch.empty_like(x) if need[0] else None
        dw = torch.empty(C, dtype=pdtype, device=x.device) if need[1] else None
        db = torch.empty(C, dtype=pdtype, device=x.device) if need[2] else None
    _check(load_library().ue5m3_layer_norm_grad(_ptr(x), _ptr(dy), rows, C, _TYPES[x.dtype], _ptr(weight), pt,
                                                _ptr(mean), _ptr(rstd), _ptr(residual_grad), _ptr(dx), _ptr(dw),
                                                _ptr(db), _stream(stream)), "ue5m3_layer_norm_grad")
    return dx, dw, db


# ---------------------------------------------------------------- dropout --
def dropout_forward(x, p, seed, tensor_id=0, residual=None, out=None, stream=None):
    """[residual +] dropout of ``x`` (bf16, fp16 or fp32) with the mask of
    (seed, tensor_id) (see ue5m3_dropout).  The same call on a gradient is
    the backward pass.  ``out`` may be ``x`` or ``residual``."""
    _tensor(x, "x", _TYPES)
    _like(residual, x, "residual")
    with _on(stream):
        y = torch.empty_like(x) if out is None else _like(out, x, "out")
    _check(load_library().ue5m3_dropout(_ptr(x), x.numel(), _TYPES[x.dtype], float(p), int(seed) & (2**64 - 1),
                                        int(tensor_id) & 0xFFFFFFFF, _ptr(residual), _ptr(y), _stream(stream)),
           "ue5m3_dropout")
    return y


# --------------------------------------------------- 8-bit floating point --
def _pair(R, C, fmt, scale, like):
    return (torch.empty((R, pad128(C)), dtype=FP8[fmt], device=like.device),
            torch.empty((pad128(C) // 128, scale_pitch(R)), dtype=SCALE[scale], device=like.device))


def _quantize(x, fmt, scale, rows, cols, stream):
    R, C = x.shape
    pr, sr = rows if rows is not None else (None, None)
    pc, sc = cols if cols is not None else (None, None)
    _check(load_library().ue5m3_quantize_fp8(_ptr(x), R, C, _TYPES[x.dtype], _FP8_CODES[FP8[fmt]],
                                             _SCALE_CODES[SCALE[scale]], _ptr(pr), _ptr(sr), _ptr(pc), _ptr(sc),
                                             _stream(stream)), "ue5m3_quantize_fp8")


def _formats(fmt, scale):
    if fmt not in FP8:
        raise ValueError(f"fmt must be one of {sorted(FP8)}")
    if scale not in SCALE:
        raise ValueError(f"scale must be one of {sorted(SCALE)}")


def quantize_fp8(x, axis, fmt="e4m3", scale="e8m0", stream=None):
    """Quantizes ``x`` [R, C] (bf16, fp16 or fp32) in blocks of 128 along its
    rows (axis 1) or down its columns (axis 0, stored transposed); see
    ue5m3_quantize_fp8.  Returns (payload, scales)."""
    _tensor(x, "x", _TYPES, dim=2)
    _formats(fmt, scale)
    if axis not in (0, 1):
        raise ValueError("axis must be 0 or 1")
    R, C = x.shape
    with _on(stream):
        out = _pair(R, C, fmt, scale, x) if axis == 1 else _pair(C, R, fmt, scale, x)
    _quantize(x, fmt, scale, out if axis == 1 else None, out if axis == 0 else None, stream)
    return out


def quantize_fp8_dual(x, fmt="e4m3", scale="e8m0", stream=None):
    """Both blockings of ``x`` from one read: ((payload, scales) of axis 1,
    (payload, scales) of axis 0), as ``quantize_fp8`` gives them."""
    _tensor(x, "x", _TYPES, dim=2)
    _formats(fmt, scale)
    R, C = x.shape
    with _on(stream):
        rows, cols = _pair(R, C, fmt, scale, x), _pair(C, R, fmt, scale, x)
    _quantize(x, fmt, scale, rows, cols, stream)
    return rows, cols


def quantize_fp8_tiles(w, scale="e8m0", transposed=True, stream=None):
    """Quantizes a weight ``w`` [R, C] to E4M3 in 128 x 128 tiles (see
    ue5m3_quantize_fp8_tiles).  Returns (payload, scales, payload_t, scales_t),
    the last two None unless ``transposed``."""
    _tensor(w, "w", _TYPES, dim=2)
    _formats("e4m3", scale)
    R, C = w.shape
    rb, cb = pad128(R) // 128, pad128(C) // 128

    def empty(shape, dtype):
        return torch.empty(shape, dtype=dtype, device=w.device)
    with _on(stream):
        p, s = empty((R, 128 * cb), FP8["e4m3"]), empty((rb, cb), SCALE[scale])
        pt, st = (empty((C, 128 * rb), FP8["e4m3"]), empty((cb, rb), SCALE[scale])) if transposed else (None, None)
    _check(load_library().ue5m3_quantize_fp8_tiles(_ptr(w), R, C, _TYPES[w.dtype], _SCALE_CODES[SCALE[scale]], _ptr(p),
                                                   _ptr(s), _ptr(pt), _ptr(st), _stream(stream)),
           "ue5m3_quantize_fp8_tiles")
    return p, s, pt, st


def _operand(p, s, rows, K, tiled, dtypes, name):
    """An 8-bit operand: ``rows`` payload rows over a contraction of K."""
    _tensor(p, name, dtypes)
    _tensor(s, name + "_scales", _SCALE_CODES)
    _dev_buf(p, p.dtype, rows * pad128(K), name)
    blocks = pad128(K) // 128
    _dev_buf(s, s.dtype, blocks * (pad128(rows) // 128 if tiled else scale_pitch(rows)), name + "_scales")


def gemm_fp8(layout, M, N, K, a, a_scales, b, b_scales, out=None, out_dtype=torch.bfloat16, a_blk=None, b_blk=None,
             stream=None):
    """C [M, N] from 8-bit operands with a scale for each block of 128 along
    the contraction (see ue5m3_gemm_fp8); layout is "nt", "nn" or "tn" as for
    ``gemm``.  ``a`` E4M3 or E5M2, ``b`` E4M3; ``a_blk`` / ``b_blk`` "row",
    "colT" or "tile" (None: activations and gradients 1D, weights in tiles, as
    each product of a linear layer has them).  The matrix instructions truncate
    small products next to large ones, at 2^-13 of those: fp32 output is 4e-5 to
    7e-5 from the exact sum in relative L2 norm on normal values."""
    lay = _LAYOUTS[layout] if isinstance(layout, str) else int(layout)
    M, N, K = int(M), int(N), int(K)
    a_blk = ("colT" if lay == TN else "row") if a_blk is None else a_blk
    b_blk = ("colT" if lay == TN else "tile") if b_blk is None else b_blk
    if M > 0 and N > 0 and K > 0:
        _operand(a, a_scales, M, K, False, _FP8_CODES, "a")
        _operand(b, b_scales, N, K, b_blk == "tile", (torch.float8_e4m3fn,), "b")
        if a_scales.dtype != b_scales.dtype:
            raise ValueError("the scales of both operands must be of one kind")
    if out is None:
        with _on(stream):
            out = torch.empty((M, N), dtype=out_dtype, device=a.device)
    if out.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("out must be fp32 or bf16")
    _dev_buf(out, out.dtype, M * N, "out")
    _check(load_library().ue5m3_gemm_fp8(lay, M, N, K, _ptr(a), _ptr(a_scales), _BLOCKINGS[a_blk],
                                         _FP8_CODES[a.dtype], _ptr(b), _ptr(b_scales), _BLOCKINGS[b_blk],
                                         _SCALE_CODES[b_scales.dtype], _ptr(out),
                                         OUT_BF16 if out.dtype == torch.bfloat16 else OUT_F32, _stream(stream)),
           "ue5m3_gemm_fp8")
    return out


def linear_fp8(x, w, w_scales, out=None, out_dtype=torch.bfloat16, stream=None):
    """Serving call: ``x`` [..., K] (bf16) times a weight [N, K] quantized once
    by ``quantize_fp8_tiles`` (``w`` [N, pad(K)], ``w_scales``); see
    ue5m3_linear_fp8.  Returns [..., N], with ``gemm_fp8``'s arithmetic."""
    _tensor(x, "x", (torch.bfloat16,))
    _tensor(w, "w", (torch.float8_e4m3fn,), x, 2)
    _tensor(w_scales, "w_scales", _SCALE_CODES, x, 2)
    K, N = x.shape[-1], w.shape[0]
    T = x.numel() // K if K else _numel(x.shape[:-1])
    if w.shape[1] != pad128(K) or w_scales.shape != (pad128(N) // 128, pad128(K) // 128):
        raise ValueError(f"w {tuple(w.shape)} and w_scales {tuple(w_scales.shape)} do not belong to inputs of {K}")
    if out is None:
        with _on(stream):
            out = torch.empty((*x.shape[:-1], N), dtype=out_dtype, device=x.device)
    if out.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("out must be fp32 or bf16")
    _dev_buf(out, out.dtype, T * N, "out")
    _check(load_library().ue5m3_linear_fp8(_ptr(x), T, K, N, _ptr(w), _ptr(w_scales), _SCALE_CODES[w_scales.dtype],
                                           _ptr(out), OUT_BF16 if out.dtype == torch.bfloat16 else OUT_F32,
                                           _stream(stream)), "ue5m3_linear_fp8")
    return out
