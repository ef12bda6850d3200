"""Norms of queries and keys for each head and their rotation by position, in
one pass over both: with gradients, and in a serving form that writes keys and
values into the pages of a cache.

Either part may be left out (``eps=None``: no norm; ``freqs=None``: no rotation).
Frequencies are a tensor of the caller's, so that any scaling for long contexts
is his; ``rotary_frequencies`` makes the common ones.
"""

import functools
import math

import torch
from torch.autograd.function import once_differentiable
from torch.autograd.graph import increment_version

from . import PagesC, RopeC, _check, _numel, _ptr, _stream, load_library
from .operators import _TYPES, recorded


def rotary_frequencies(dim, base=10000.0, factor=1.0, kind="linear", original=None, low=1.0, high=32.0, device="cuda"):
    """(freqs, amplitude) for ``qk_norm_rope``: fp32 [dim / 2], base^(-2 i / dim)
    scaled for contexts ``factor`` times as long:

      linear   all divided by ``factor``
      base     the base raised, by factor^(dim / (dim - 2)): the last frequency is
               divided by ``factor``, the first stays
      parts    divided by ``factor`` where ``original`` positions (the context
               trained on) are fewer than ``low`` turns, kept where they are more
               than ``high``, in between in proportion; the amplitude is
               0.1 ln(factor) + 1
    """
    dim = int(dim)
    if dim < 2 or dim % 2 or not base > 1.0 or not factor >= 1.0:
        raise ValueError("dim must be even and positive, base above 1, factor at least 1")
    i = torch.arange(0, dim, 2, dtype=torch.float64)
    amplitude = 1.0
    if kind == "base":
        if dim == 2 and factor != 1.0:
            raise ValueError("one pair has no base to raise")
        f = (base * factor ** (dim / max(dim - 2, 1))) ** (-i / dim)
    else:
        f = base ** (-i / dim)
        if kind == "linear":
            f = f / factor
        elif kind == "parts":
            if original is None or not 0 < low < high:
                raise ValueError("parts needs the original context and 0 < low < high")
            turns = original * f / (2 * math.pi)
            keep = ((turns - low) / (high - low)).clamp(0.0, 1.0)
            f = f * (keep + (1.0 - keep) / factor)
            amplitude = 0.1 * math.log(factor) + 1.0
        else:
            raise ValueError("kind must be linear, base or parts")
    return f.float().to(device), amplitude


def packed_positions(starts, tokens):
    """Position of each of ``tokens`` tokens in its own sequence, of sequences packed one
    after the other from ``starts``[i] on (int64, on their device)."""
    at = torch.arange(tokens, dtype=torch.int64, device=starts.device)
    starts = starts.to(torch.int64)
    i = torch.searchsorted(starts, at, right=True) - 1
    return at - starts[i.clamp_min(0)]


def _on_device(t, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA/HIP tensor")
    if t.get_device() != torch._C._cuda_getDevice():
        raise ValueError(f"{name} is on {t.device}, not on the device of the call")
    return t


# (small calls are bound by the host: what follows from shapes and strides is worked out
# once for each)
@functools.lru_cache(maxsize=4096)
def _row_layout(shape, stride, dense):
    """(tokens, token stride, head stride) of [..., heads, dim], None where a copy is
    needed for them.  Of one token, or one head, the stride reaches nothing and may be any
    number: 0 then."""
    ok = stride[-1] == 1 or shape[-1] == 1
    token, tokens = stride[-3], _numel(shape[:-2])
    for d in range(len(shape) - 4, -1, -1):              # leading dimensions as one
        if shape[d] > 1:
            inner = _numel(shape[d + 1:-2])
            ok = ok and (inner <= 1 or stride[d] == token * inner)
            if inner <= 1:
                token = stride[d]
    token, head = token if tokens > 1 else 0, stride[-2] if shape[-2] > 1 else 0
    if dense:
        ok = (ok and (tokens <= 1 or shape[-1] <= token < 1 << 23) and (shape[-2] <= 1 or head >= shape[-1])
              and token % 8 == 0 and head % 8 == 0)
    return (tokens, token, head) if ok else None


def head_rows(t, name, dtypes=_TYPES, dense=False):
    """``t`` [..., heads, dim] as (tensor, tokens, token stride, head stride): itself
    where its strides allow, with the elements of a head together, else a copy.
    ``dense``: as the attention kernels take it (heads apart, 16-byte aligned)."""
    _on_device(t, name)
    shape = t.shape
    if t.dtype not in dtypes or len(shape) < 3:
        raise ValueError(f"{name} must be [..., tokens, heads, dim] of " + ", ".join(str(d) for d in dtypes))
    layout = _row_layout(shape, t.stride(), dense)
    if layout is None or dense and t.data_ptr() % 16:
        t = dense_like(t).copy_(t)                   # (a clone of a contiguous tensor would keep its strides)
        layout = _row_layout(shape, t.stride(), False)
    return (t, *layout)


def dense_like(t):
    """An uninitialised dense tensor of t's shape and type (1.2 us; torch.empty of them 2.3)."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _vector(t, name, dtypes, n):
    if t is None:
        return None
    _on_device(t, name)
    if t.dtype not in dtypes or t.dim() != 1 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous vector of {n} of " + ", ".join(str(d) for d in dtypes))
    return t


@functools.lru_cache(maxsize=1024)
def _template(q_shape, q_layout, k_shape, k_layout, dtype, wt, pairs, norm, interleaved):
    """A RopeC without its addresses, eps and amplitude, as bytes: sizes, types, strides, and
    dense outputs (an append of one token 18.5 us, with all fields set in each call 19.9)."""
    dim, q_heads, kv_heads = k_shape[-1], q_shape[-2] if q_shape is not None else 0, k_shape[-2]
    _, q_token, q_head = q_layout if q_layout is not None else (0, 0, 0)
    tokens, k_token, k_head = k_layout
    return bytes(RopeC(tokens, q_heads, kv_heads, dim, pairs, _TYPES[dtype], _TYPES[wt], norm, interleaved, 0.0, 1.0, None, None,
                       q_token, q_head, k_token, k_head, None, None, None, max(int(k_shape[-3]), 1), None, None, None,
                       q_heads * dim, dim, kv_heads * dim, dim))


def _arguments(q, k, q_weight, k_weight, positions, freqs, eps, interleaved, amplitude):
    """A RopeC of all but the outputs' addresses, and the tensors that it points to."""
    kr, *k_layout = head_rows(k, "k")
    shape, dtype = k.shape, k.dtype
    lead, dim = shape[:-2], shape[-1]
    qr = q_shape = q_layout = None
    if q is not None:
        qr, *q_layout = head_rows(q, "q")
        q_shape = q.shape
        if q_shape[:-2] != lead or q_shape[-1] != dim or q.dtype != dtype:
            raise ValueError(f"q {tuple(q_shape)} and k {tuple(shape)} must have the same tokens, head size and type")
        q_layout = tuple(q_layout)
    if not 1 <= dim <= 256:
        raise ValueError("heads have 1 to 256 elements")
    norm, wt = eps is not None, dtype
    if q_weight is not None or k_weight is not None:
        if not norm:
            raise ValueError("weights belong to the norm: pass eps")
        wt = (k_weight if q_weight is None else q_weight).dtype
        types = (wt,) if wt in (dtype, torch.float32) else (dtype, torch.float32)
        _vector(q_weight, "q_weight", types, dim)
        _vector(k_weight, "k_weight", types, dim)
    pairs = 0
    if freqs is not None:
        pairs = freqs.numel()
        _vector(freqs, "freqs", (torch.float32,), pairs)
        if freqs.requires_grad:
            raise ValueError("freqs have no gradient")
        if not 1 <= pairs <= dim // 2:
            raise ValueError(f"{pairs} frequencies for heads of {dim}")
        if positions is not None:
            _on_device(positions, "positions")
            if positions.dtype not in (torch.int64, torch.int32):
                raise ValueError("positions must be integers")
            if positions.dtype != torch.int64 or positions.shape != lead or not positions.is_contiguous():
                positions = positions.to(torch.int64).expand(lead).contiguous()
    else:
        positions = None
    args = RopeC.from_buffer_copy(_template(q_shape, q_layout, shape, tuple(k_layout), dtype, wt, pairs, int(norm),
                                            int(bool(interleaved))))
    args.eps, args.amplitude = float(eps) if norm else 0.0, float(amplitude)
    args.q, args.k, args.q_weight, args.k_weight = _ptr(qr), _ptr(kr), _ptr(q_weight), _ptr(k_weight)
    args.positions, args.freqs = _ptr(positions), _ptr(freqs)
    return args, (qr, kr, positions)


def _forward(q, k, *rest):
    args, kept = _arguments(q, k, *rest)
    q_out, k_out = dense_like(q), dense_like(k)
    args.q_out, args.k_out = q_out.data_ptr(), k_out.data_ptr()
    _check(load_library().ue5m3_qk_norm_rope(args, _stream()), "ue5m3_qk_norm_rope")
    return q_out, k_out, kept


class _RopeFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, positions, freqs, eps, interleaved, amplitude):
        q_out, k_out, (qr, kr, positions) = _forward(q, k, q_weight, k_weight, positions, freqs, eps, interleaved, amplitude)
        norm = eps is not None
        ctx.save_for_backward(qr if norm else None, kr if norm else None, q_weight, k_weight, positions, freqs)
        ctx.rest, ctx.shapes = (eps, interleaved, amplitude), (q.shape, k.shape)
        ctx.set_materialize_grads(False)
        return q_out, k_out

    @staticmethod
    @once_differentiable
    def backward(ctx, gq, gk):
        q, k, q_weight, k_weight, positions, freqs = ctx.saved_tensors
        if gq is None and gk is None:
            return (None,) * 9
        like = gq if gq is not None else gk
        gq, gk = (torch.zeros(s, dtype=like.dtype, device=like.device) if g is None else g.contiguous()
                  for g, s in zip((gq, gk), ctx.shapes))
        # (without the norm the inputs do not matter: the gradients stand in for them)
        args, kept = _arguments(gq if q is None else q, gk if k is None else k, q_weight, k_weight, positions, freqs, *ctx.rest)
        need_q, need_k, need_qw, need_kw = ctx.needs_input_grad[:4]
        new = lambda t, need: dense_like(t) if need else None  # noqa: E731
        dq, dk = new(gq, need_q), new(gk, need_k)
        dqw, dkw = new(q_weight, need_qw and q_weight is not None), new(k_weight, need_kw and k_weight is not None)
        args.q_out, args.k_out = _ptr(dq), _ptr(dk)
        lib, scratch = load_library(), None
        if dqw is not None or dkw is not None:
            n = lib.ue5m3_qk_norm_rope_grad_scratch(args.tokens, args.q_heads + args.kv_heads, args.dim)
            scratch = torch.empty(n, dtype=torch.uint8, device=like.device)
        _check(lib.ue5m3_qk_norm_rope_grad(args, gq.data_ptr(), gk.data_ptr(), _ptr(dqw), _ptr(dkw), _ptr(scratch), _stream()),
               "ue5m3_qk_norm_rope_grad")
        return dq, dk, dqw, dkw, None, None, None, None, None


def qk_norm_rope(q, k, q_weight=None, k_weight=None, positions=None, freqs=None, eps=1e-6, interleaved=False,
                 amplitude=1.0):
    """Queries ``q`` [..., L, heads, dim] and keys ``k`` [..., L, kv_heads, dim] (bf16,
    fp16 or fp32; strided views of one projection's output are fine) normed over each
    head, times ``q_weight`` and ``k_weight`` [dim] (of their type or fp32, or None), and
    rotated by position, with gradients (see ue5m3_qk_norm_rope).

    ``freqs``: fp32, one for each rotated pair: the first 2 len(freqs) elements of a
    head turn, in halves (i with i + len(freqs)) or, ``interleaved``, neighbours
    together.  ``positions``: integers [..., L], broadcast over leading dimensions
    (None: 0 .. L - 1 in each).  The weights' gradients are summed in fp32 in a fixed
    order.  Returns new dense tensors (q, k)."""
    if recorded(q, k, q_weight, k_weight, freqs):
        return _RopeFn.apply(q, k, q_weight, k_weight, positions, freqs, eps, bool(interleaved), float(amplitude))
    return _forward(q, k, q_weight, k_weight, positions, freqs, eps, interleaved, amplitude)[:2]


@functools.lru_cache(maxsize=1024)
def _page_layout(shape, stride, multiple):
    if len(shape) != 4 or stride[3] != 1 and shape[3] > 1:
        raise ValueError("a cache must be [pages, page_size, kv_heads, dim], a head's elements together")
    size = shape[1]
    if size < 1 or size & (size - 1):
        raise ValueError("pages hold a power of two of tokens")
    strides = [s if n > 1 else 0 for n, s in zip(shape[:3], stride)]     # (of one page, token or head: it reaches nothing)
    if any(s % multiple for s in strides):
        raise ValueError(f"the cache's strides must be multiples of {multiple} elements")
    return (shape[0], size, *strides)


def cache_arguments(k_cache, v_cache, multiple=1):
    """PagesC of the keys and values [pages, page_size, kv_heads, dim] of one layer."""
    _on_device(k_cache, "k_cache")
    _on_device(v_cache, "v_cache")
    shape, stride = k_cache.shape, k_cache.stride()
    layout = _page_layout(shape, stride, multiple)
    if (shape != v_cache.shape or k_cache.dtype != v_cache.dtype or
            stride != v_cache.stride() and layout != _page_layout(shape, v_cache.stride(), multiple)):
        raise ValueError("k_cache and v_cache must have one shape, type and strides")
    return PagesC(k_cache.data_ptr(), v_cache.data_ptr(), *layout)


def qk_norm_rope_append(q, k, v, k_cache, v_cache, slots, q_weight=None, k_weight=None, positions=None, freqs=None,
                        eps=1e-6, interleaved=False, amplitude=1.0):
    """The serving form of ``qk_norm_rope``: returns the queries, and writes the keys,
    normed and rotated, and the values ``v`` into a cache (``k_cache``, ``v_cache``
    [pages, page_size, kv_heads, dim], any strides with a head's elements together), token
    t at ``slots``[t] (int64) = page * page_size + place, no two at one (see
    ue5m3_qk_norm_rope_append).  A slot below 0 or past the cache writes nothing.
    ``q`` may be None (keys that are ready: with eps=None and no freqs they are
    copied); then None is returned."""
    if recorded(q, k, v, q_weight, k_weight, freqs, k_cache, v_cache):
        raise RuntimeError("qk_norm_rope_append has no gradients: call it under torch.no_grad()")
    args, kept = _arguments(q, k, q_weight, k_weight, positions, freqs, eps, interleaved, amplitude)
    vr, tokens, v_token, v_head = head_rows(v, "v")
    if v.shape != k.shape or v.dtype != k.dtype:
        raise ValueError(f"v {tuple(v.shape)} must have the shape and type of k {tuple(k.shape)}")
    cache = cache_arguments(k_cache, v_cache)
    if k_cache.shape[2:] != k.shape[-2:] or k_cache.dtype != k.dtype:
        raise ValueError(f"a cache of {tuple(k_cache.shape)} {k_cache.dtype} does not take keys of {tuple(k.shape)} {k.dtype}")
    _on_device(slots, "slots")
    if slots.dtype != torch.int64 or slots.numel() != tokens or not slots.is_contiguous():
        raise ValueError(f"slots must be {tokens} contiguous int64 numbers")
    q_out = None if q is None else dense_like(q)
    args.q_out = _ptr(q_out)
    _check(load_library().ue5m3_qk_norm_rope_append(args, vr.data_ptr(), v_token, v_head, cache, slots.data_ptr(), _stream()),
           "ue5m3_qk_norm_rope_append")
    increment_version((k_cache, v_cache))            # (autograd finds out where it has saved them)
    return q_out
