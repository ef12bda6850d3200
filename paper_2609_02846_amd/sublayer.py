"""Pre-norm residual branches: x + dropout(linear(layer_norm(x))) in training, layer
norm, the 8-bit linear layer and dropout together; and the attention branch, in
training and over a paged cache.

The first is one autograd function, so that what the branch's ends share is joined: the
residual is added in dropout's pass, and its gradient in the norm's backward
pass.  Between the operators bf16 tensors are handed on, as between the
separate calls, and the results are theirs.
"""

import torch
from torch.autograd.function import once_differentiable

from . import _check, _stream, load_library
from .attention import attention, paged_attention
from .dropout import Dropout
from .fp8 import Fp8Linear, _check_formats, _flat, backward_products, forward_product
from .norm import LayerNorm
from .operators import BF16, dropout_forward, layer_norm_forward, norm_args, recorded
from .rotary import packed_positions, qk_norm_rope, qk_norm_rope_append, rotary_frequencies


class _SublayerFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gain, bias, w, p, seed, tensor_id, eps, scale, grad_fmt, need_w):
        pt, T, C = norm_args(x, gain, bias)
        lib, stream = load_library(), _stream()
        h, stats = torch.empty_like(x), torch.empty(2 * T, dtype=torch.float32, device=x.device)
        mean = stats.data_ptr()
        _check(lib.ue5m3_layer_norm(x.data_ptr(), T, C, BF16, None if gain is None else gain.data_ptr(),
                                    None if bias is None else bias.data_ptr(), pt, eps, h.data_ptr(), mean, mean + 4 * T,
                                    stream), "ue5m3_layer_norm")
        y, keep = forward_product(h, w, scale, True, need_w)
        _check(lib.ue5m3_dropout(y.data_ptr(), T * C, BF16, p, seed, tensor_id, x.data_ptr(), y.data_ptr(), stream),
               "ue5m3_dropout")
        ctx.save_for_backward(x, gain, stats, keep)
        ctx.args = (T, C, C, scale, grad_fmt, True, need_w)
        ctx.key, ctx.pt = (p, seed, tensor_id), pt
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        x, gain, stats, keep = ctx.saved_tensors
        need_x, need_g, need_b = ctx.needs_input_grad[:3]
        T, C = ctx.args[:2]
        lib, stream = load_library(), _stream()
        dout = dout.to(torch.bfloat16).contiguous()
        dy, dev = torch.empty_like(dout), x.device
        _check(lib.ue5m3_dropout(dout.data_ptr(), T * C, BF16, *ctx.key, None, dy.data_ptr(), stream), "ue5m3_dropout")
        dh, dw = backward_products(dy, keep, *ctx.args)
        pdtype = torch.bfloat16 if ctx.pt == BF16 else torch.float32
        dx = dy if need_x else None                  # dropout's gradient has been read
        dg = torch.empty(C, dtype=pdtype, device=dev) if need_g else None
        db = torch.empty(C, dtype=pdtype, device=dev) if need_b else None
        mean = stats.data_ptr()
        _check(lib.ue5m3_layer_norm_grad(x.data_ptr(), dh.data_ptr(), T, C, BF16, None if gain is None else gain.data_ptr(),
                                         ctx.pt, mean, mean + 4 * T, dout.data_ptr(), dx.data_ptr() if need_x else None,
                                         dg.data_ptr() if need_g else None, db.data_ptr() if need_b else None, stream),
               "ue5m3_layer_norm_grad")
        return dx, dg, db, dw, None, None, None, None, None, None, None


def sublayer(x, gain, bias, weight, p=0.1, seed=0, tensor_id=0, eps=1e-5, scale="e8m0", grad_fmt="e4m3"):
    """x + dropout(fp8_linear(layer_norm(x, gain, bias), weight)) for bf16
    ``x`` [..., C] and ``weight`` [C, C], with gradients."""
    _check_formats(scale, grad_fmt)
    C = x.shape[-1]
    if tuple(weight.shape) != (C, C):
        raise ValueError(f"the branch's weight must be [{C}, {C}] to add to its input")
    x2 = _flat(x, C)
    if recorded(x2, gain, bias, weight):
        y = _SublayerFn.apply(x2, gain, bias, weight, float(p), int(seed) & (2 ** 64 - 1), int(tensor_id) & 0xFFFFFFFF,
                              float(eps), scale, grad_fmt, weight.requires_grad)
    else:
        h = layer_norm_forward(x2, gain, bias, eps)
        y, _ = forward_product(h, weight, scale, False, False)
        y = dropout_forward(y, p, seed, tensor_id, residual=x2, out=y)
    return y if x.dim() == 2 else y.reshape(x.shape)


class PreNormSublayer(torch.nn.Module):
    """The branch with its parameters.  In evaluation dropout passes and, after
    ``linear.freeze()``, the product takes the quantized weight.  ``seed`` and
    ``layer_id`` are dropout's (see ``Dropout``)."""

    def __init__(self, features, p=0.1, eps=1e-5, scale="e8m0", grad_fmt="e4m3", seed=None, layer_id=0, device="cuda"):
        super().__init__()
        self.norm = LayerNorm(features, eps, device=device)
        self.linear = Fp8Linear(features, features, scale, grad_fmt, device)
        self.dropout = Dropout(p, seed, layer_id)

    def forward(self, x):
        if not self.training or self.linear.frozen is not None:
            return self.dropout(self.linear(self.norm(x)), residual=x)
        d = self.dropout
        return sublayer(x, self.norm.weight, self.norm.bias, self.linear.weight, d.p, d.next_key(), d.layer_id,
                        self.norm.eps, self.linear.scale, self.linear.grad_fmt)


class PreNormAttention(torch.nn.Module):
    """The attention branch of a decoder layer,

        x + dropout(out(attention(norm_rope(qkv(layer_norm(x)))))),

    with 8-bit linear layers (see ``Fp8Linear``), norms of queries and keys over each
    head, rotation by position, and causal attention with an optional ``window`` and
    ``sinks``.  ``rotary``: (freqs, amplitude), as ``rotary_frequencies`` gives them (None:
    its defaults for the whole head).

    ``forward`` is for training and evaluation of whole sequences; ``prompt`` is the same
    without gradients and fills a cache; ``token`` takes one new token of each of several
    sequences."""

    def __init__(self, features, q_heads, kv_heads, head_dim, p=0.1, eps=1e-5, qk_eps=1e-6, rotary=None, window=0, sinks=0,
                 scale="e8m0", grad_fmt="e4m3", seed=None, layer_id=0, device="cuda"):
        super().__init__()
        if q_heads < 1 or kv_heads < 1 or q_heads % kv_heads:
            raise ValueError(f"{q_heads} query heads cannot share {kv_heads} key-value heads evenly")
        self.heads, self.head_dim = (int(q_heads), int(kv_heads), int(kv_heads)), int(head_dim)
        self.qk_eps, self.window, self.sinks = float(qk_eps), int(window), int(sinks)
        self.norm = LayerNorm(features, eps, device=device)
        self.qkv = Fp8Linear(features, sum(self.heads) * head_dim, scale, grad_fmt, device)
        self.out = Fp8Linear(q_heads * head_dim, features, scale, grad_fmt, device)
        self.q_weight, self.k_weight = (torch.nn.Parameter(torch.ones(head_dim, dtype=torch.bfloat16, device=device))
                                        for _ in range(2))
        self.dropout = Dropout(p, seed, layer_id)
        freqs, self.amplitude = rotary_frequencies(head_dim, device=device) if rotary is None else rotary
        self.register_buffer("freqs", freqs, persistent=False)

    def _apply(self, fn, recurse=True):
        freqs = self.freqs
        super()._apply(fn, recurse)
        if self.freqs.dtype != torch.float32:        # (moved with the module, not cast with it)
            self.freqs = freqs.to(self.freqs.device)
        return self

    def _rotary(self, positions):
        return self.q_weight, self.k_weight, positions, self.freqs, self.qk_eps, False, self.amplitude

    def _project(self, x):
        qkv = self.qkv(self.norm(x))
        return qkv.view(*x.shape[:-1], sum(self.heads), self.head_dim).split(self.heads, dim=-2)

    def _close(self, o, x):
        return self.dropout(self.out(o.reshape(*x.shape[:-1], self.heads[0] * self.head_dim)), residual=x)

    def _attend(self, x, starts, positions):
        q, k, v = self._project(x)
        if positions is None and starts is not None:
            positions = packed_positions(starts, x.shape[0])
        q, k = qk_norm_rope(q, k, *self._rotary(positions))
        return self._close(attention(q, k, v, starts, window=self.window, sinks=self.sinks), x), k, v

    def forward(self, x, starts=None, positions=None):
        """``x`` [batch, length, features] (bf16), or [tokens, features] of sequences packed
        one after the other (``starts``, as ``attention`` takes them).  ``positions`` default
        to each sequence's own, from 0."""
        return self._attend(x, starts, positions)[0]

    @torch.no_grad()
    def prompt(self, x, k_cache, v_cache, slots, starts=None, positions=None):
        """``forward`` of whole prompts [tokens, features], whose keys and values go to
        ``slots`` of a cache (see ``qk_norm_rope_append``)."""
        y, k, v = self._attend(x, starts, positions)
        qk_norm_rope_append(None, k, v, k_cache, v_cache, slots, eps=None)
        return y

    @torch.no_grad()
    def token(self, x, k_cache, v_cache, slots, table, lengths):
        """One new token of each of several sequences, ``x`` [rows, features]: its key and
        value go to ``slots``, and it attends to the ``lengths`` tokens of its row of
        ``table``, itself the last (see ``paged_attention``)."""
        q, k, v = self._project(x)
        q = qk_norm_rope_append(q, k, v, k_cache, v_cache, slots, *self._rotary(lengths - 1))
        return self._close(paged_attention(q, k_cache, v_cache, table, lengths, window=self.window, sinks=self.sinks), x)
