"""Attention of ragged sequences, causal, with a sliding window and first tokens
that stay visible, with gradients; and attention of single tokens over a paged
cache."""

import torch
from torch.autograd.function import once_differentiable

from . import AttentionC, AttentionGradC, PagedAttentionC, _check, _numel, _ptr, _stream, load_library
from .operators import _TYPES, recorded
from .rotary import _on_device, cache_arguments, dense_like, head_rows

_HALF = (torch.bfloat16, torch.float16)


def _starts(t, name):
    if t is None:
        return None
    _on_device(t, name)
    if t.dtype != torch.int32 or t.dim() != 1 or t.numel() < 2 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 vector of at least two numbers")
    return t


def _span(n):
    """A window or a number of sinks: what passes every length stands for that (as an int64
    it would come round)."""
    return min(int(n), 1 << 62)


def _heads(q_heads, kv_heads, dim, window, sinks):
    if q_heads < 1 or kv_heads < 1 or q_heads % kv_heads:
        raise ValueError(f"{q_heads} query heads cannot share {kv_heads} key-value heads evenly")
    if dim % 8 or not 8 <= dim <= 128:
        raise ValueError("heads have a multiple of 8 elements, up to 128")
    if window < 0 or sinks < 0:
        raise ValueError("window and sinks must not be negative")


def _arguments(q, k, v, q_starts, k_starts, scale, causal, window, sinks):
    """An AttentionC of all but the outputs, and the tensors that it points to."""
    qr, q_tokens, q_token, q_head = head_rows(q, "q", _HALF, True)
    kr, k_tokens, k_token, k_head = head_rows(k, "k", _HALF, True)
    vr, _, v_token, v_head = head_rows(v, "v", _HALF, True)
    if k.shape != v.shape or not q.dtype == k.dtype == v.dtype or q.shape[-1] != k.shape[-1] or q.dim() != k.dim():
        raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)} and v {tuple(v.shape)} do not belong together")
    q_starts, k_starts = _starts(q_starts, "q_starts"), _starts(k_starts, "k_starts")
    if q_starts is None:
        if k_starts is not None:
            raise ValueError("k_starts without q_starts")
        if q.dim() > 3 and q.shape[:-3] != k.shape[:-3]:
            raise ValueError(f"q {tuple(q.shape)} and k {tuple(k.shape)} are batches of different sizes")
        sequences = _numel(q.shape[:-3])
    else:
        if q.dim() != 3:
            raise ValueError("ragged sequences come as [tokens, heads, dim]")
        if k_starts is None:
            if k_tokens != q_tokens:
                raise ValueError("k_starts is needed where there are more or fewer keys than queries")
            k_starts = q_starts
        if k_starts.numel() != q_starts.numel():
            raise ValueError("q_starts and k_starts must name the same number of sequences")
        sequences = q_starts.numel() - 1
    window, sinks = _span(window), _span(sinks)
    _heads(q.shape[-2], k.shape[-2], q.shape[-1], window, sinks)
    if window and not causal:
        raise ValueError("a window belongs to causal attention")
    scale = q.shape[-1] ** -0.5 if scale is None else float(scale)
    args = AttentionC(q_tokens, k_tokens, max(sequences, 1), _ptr(q_starts), _ptr(k_starts), q.shape[-2], k.shape[-2],
                      q.shape[-1], _TYPES[q.dtype], int(bool(causal)), scale, window, sinks, qr.data_ptr(), kr.data_ptr(),
                      vr.data_ptr(), q_token, q_head, k_token, k_head, v_token, v_head)
    return args, (qr, kr, vr, q_starts, k_starts)


def attention_forward(q, k, v, q_starts=None, k_starts=None, scale=None, causal=True, window=0, sinks=0, lse=False,
                      _rest=False):
    """``attention`` without gradients; with ``lse`` (o, lse): the fp32 logarithms of
    the rows' sums [heads, tokens]."""
    args, kept = _arguments(q, k, v, q_starts, k_starts, scale, causal, window, sinks)
    o = dense_like(q)
    sums = torch.empty((args.q_heads, args.q_tokens), dtype=torch.float32, device=q.device) if lse else None
    args.o, args.lse = o.data_ptr(), _ptr(sums)
    rest = None
    if _rest:
        rest = dense_like(o)
        args.o_rest = rest.data_ptr()
    lib = load_library()
    n = lib.ue5m3_attention_scratch(args)
    scratch = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
    _check(lib.ue5m3_attention(args, _ptr(scratch), _stream()), "ue5m3_attention")
    return (o, sums, rest) if _rest else (o, sums) if lse else o


class _AttentionFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, q_starts, k_starts, *rest):
        o, lse, o_rest = attention_forward(q, k, v, q_starts, k_starts, *rest, lse=True, _rest=True)
        ctx.save_for_backward(q, k, v, q_starts, k_starts, o, o_rest, lse)
        ctx.rest = rest
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, do):
        q, k, v, q_starts, k_starts, o, o_rest, lse = ctx.saved_tensors
        need_q, need_k, need_v = ctx.needs_input_grad[:3]
        args, kept = _arguments(q, k, v, q_starts, k_starts, *ctx.rest)
        args.o, args.o_rest, args.lse = o.data_ptr(), o_rest.data_ptr(), lse.data_ptr()
        do = do.contiguous()
        if do.data_ptr() % 16:
            do = do.clone()
        dq = dense_like(q) if need_q else None
        dk, dv = (dense_like(k), dense_like(v)) if need_k or need_v else (None, None)
        lib = load_library()
        scratch = torch.empty(lib.ue5m3_attention_grad_scratch(args), dtype=torch.uint8, device=lse.device)
        qs, ks, d = q.shape[-2] * q.shape[-1], k.shape[-2] * k.shape[-1], q.shape[-1]
        grad = AttentionGradC(do.data_ptr(), scratch.data_ptr(), _ptr(dq), _ptr(dk), _ptr(dv), qs, d, ks, d, ks, d)
        _check(lib.ue5m3_attention_grad(args, grad, _stream()), "ue5m3_attention_grad")
        return dq, dk if need_k else None, dv if need_v else None, None, None, None, None, None, None


def attention(q, k, v, q_starts=None, k_starts=None, scale=None, causal=True, window=0, sinks=0):
    """Softmax attention of ``q`` over ``k`` and ``v`` (bf16 or fp16; gradients: bf16),
    [batch, length, heads, dim], or [tokens, heads, dim] of sequences packed one after
    the other, sequence i from ``q_starts``[i] to ``q_starts``[i + 1] (int32; ``k_starts``
    for the keys where these differ).  Heads of queries share those of keys and values in
    equal groups, of a multiple of 8 elements up to 128.

    ``causal``: the last query of a sequence stands at its last key, and a query sees
    keys up to its own position; of these, with ``window`` > 0, the last ``window`` ones
    and the first ``sinks``.  A query that sees nothing gives zeros, as do tokens of no
    sequence.  What a query does not see may be anything (for gradients all of a sequence
    has to be finite).  ``scale``: of the scores (None: dim^-1/2).  The same call gives the
    same bits, gradients included.  See ue5m3_attention."""
    if recorded(q, k, v):
        if isinstance(q, torch.Tensor) and q.dtype == torch.float16:
            raise NotImplementedError("attention in fp16 has no gradients")
        return _AttentionFn.apply(q, k, v, q_starts, k_starts, scale, causal, window, sinks)
    return attention_forward(q, k, v, q_starts, k_starts, scale, causal, window, sinks)


def paged_attention(q, k_cache, v_cache, table, lengths, scale=None, window=0, sinks=0):
    """Attention of one new token for each sequence: ``q`` [rows, heads, dim] (bf16 or
    fp16) over the caches [pages, page_size, kv_heads, dim] (any strides of a multiple of
    8, a head's elements together).  Row i has ``lengths``[i] tokens (int32; its new one
    is the last, already in the cache) on the pages ``table``[i] (int32 [rows, width]).
    ``window`` and ``sinks`` as in ``attention``.  A row of no tokens gives zeros; one that
    needs a page outside the cache, or more pages than the table has, gives NaN.  See
    ue5m3_paged_attention."""
    if recorded(q, k_cache, v_cache):
        raise RuntimeError("paged_attention has no gradients: call it under torch.no_grad()")
    qr, rows, q_token, q_head = head_rows(q, "q", _HALF, True)
    if q.dim() != 3:
        raise ValueError("q must be [rows, heads, dim]")
    cache = cache_arguments(k_cache, v_cache, 8)
    if k_cache.shape[3] != q.shape[2] or k_cache.dtype != q.dtype:
        raise ValueError(f"a cache of {tuple(k_cache.shape)} {k_cache.dtype} does not belong to queries of "
                         f"{tuple(q.shape)} {q.dtype}")
    if k_cache.data_ptr() % 16 or v_cache.data_ptr() % 16:
        raise ValueError("the caches must be 16-byte aligned")
    for t, name in ((table, "table"), (lengths, "lengths")):
        _on_device(t, name)
        if t.dtype != torch.int32 or t.dim() != (2 if t is table else 1) or t.shape[0] != rows:
            raise ValueError(f"{name} must be int32 with {rows} rows")
    if table.stride(1) != 1 and table.shape[1] > 1 or rows > 1 and table.stride(0) < table.shape[1]:
        table = table.contiguous()
    lengths = lengths.contiguous()
    width, window, sinks = table.shape[1], _span(window), _span(sinks)
    _heads(q.shape[1], k_cache.shape[2], q.shape[2], window, sinks)
    lib = load_library()
    o = dense_like(q)
    n = lib.ue5m3_paged_attention_scratch(rows, q.shape[1], k_cache.shape[2], q.shape[2], width * cache.page_size, window, sinks)
    scratch = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
    args = PagedAttentionC(rows, q.shape[1], k_cache.shape[2], q.shape[2], _TYPES[q.dtype],
                           q.shape[2] ** -0.5 if scale is None else float(scale), window, sinks, qr.data_ptr(), q_token, q_head,
                           cache, table.data_ptr(), width, table.stride(0), lengths.data_ptr(), o.data_ptr())
    _check(lib.ue5m3_paged_attention(args, _ptr(scratch), _stream()), "ue5m3_paged_attention")
    return o
