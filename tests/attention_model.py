"""Plain implementations, in 64 bits, of the operators between the QKV and the
output projection, with bounds on how far the kernels may be from them.

A rounding to a type is off by half a step, U = eps / 2 relative to the value; a
binary32 operation by 2^-24, counted twice where the matrix instructions sum."""

import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
F = 2.0 ** -24
# Below its least normal number, 2 / eps times its least one, a type's numbers are a
# fixed step apart: fp16 has ten bits after the point from 2^-14 on, so its step there
# is 2^-24 and a rounding off by up to 2^-25, however small the value (bf16: seven from
# 2^-126, 2^-133; fp32 2^-149).
STEP = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}


def rounding(y, dtype):
    """How far the rounding of y to a type may be off."""
    return U[dtype] * y.abs() + STEP[dtype] / 2


def rope(x, w, positions, freqs, eps, interleaved, amplitude):
    """(y, size): x [T, H, D] normed and rotated, and the sum of the magnitudes that
    each element of y is made of; any float64 x (differentiable)."""
    if eps is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        if w is not None:
            x = x * w
    if freqs is None:
        return x, x.abs()
    P = freqs.numel()
    theta = positions.double()[:, None, None] * freqs.double()
    c, s = torch.cos(theta) * amplitude, torch.sin(theta) * amplitude
    at = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if interleaved else (slice(0, P), slice(P, 2 * P))
    a, b = x[..., at[0]], x[..., at[1]]
    y, size = x.clone(), x.abs()
    y[..., at[0]], y[..., at[1]] = a * c - b * s, a * s + b * c
    size[..., at[0]] = size[..., at[1]] = (a.abs() + b.abs()) * abs(amplitude)
    return y, size


def rope_bound(y, size, dtype):
    # the norm: a sum of up to 256 squares in a tree of six and chains of four to
    # eight, its root, quotient and products, 24 operations at most on any path; the
    # angle's rounding, cos and sin 4; the turn 4
    return rounding(y, dtype) + 32 * F * size + 1e-38


def visible(L, S, causal=True, window=0, sinks=0, device="cuda"):
    p = torch.arange(L, device=device)[:, None] + S - L
    j = torch.arange(S, device=device)[None]
    see = torch.ones((L, S), dtype=torch.bool, device=device)
    if causal:
        see = j <= p
        if window:
            see = see & ((p - j < window) | (j < sinks))
    return see


class Sequence:
    """One sequence's attention: q [L, H, D], k and v [S, Hk, D] of any type."""

    def __init__(self, q, k, v, scale, causal=True, window=0, sinks=0):
        self.dtype, self.scale = q.dtype, scale
        L, H, D = q.shape
        S, Hk, _ = k.shape
        self.group, self.n, self.D = H // Hk, S, D
        self.q = q.double().transpose(0, 1)
        self.k, self.v = (t.double().transpose(0, 1).repeat_interleave(self.group, 0) for t in (k, v))
        see = visible(L, S, causal, window, sinks, q.device)
        s = scale * (self.q @ self.k.transpose(1, 2)) if S else self.q.new_zeros(H, L, 0)
        s = s.masked_fill(~see, -math.inf)
        top = s.amax(-1, keepdim=True) if S else s.new_full((H, L, 1), -math.inf)
        empty = top == -math.inf
        e = torch.exp(s - top.masked_fill(empty, 0.0))
        total = e.sum(-1, keepdim=True)
        self.p = e / total.masked_fill(empty, 1.0)
        self.lse = (top + torch.log(total)).squeeze(-1)
        self.o = self.p @ self.v
        # how far a score's exponent may be off, the largest of a row: its sum over
        # D, the multiplication into powers of two and what is subtracted; lse's own
        # rounding
        size = (self.q.abs() @ self.k.abs().transpose(1, 2)).masked_fill(~see, 0.0) * scale
        self.off = ((2 * D + 8) * F * size).amax(-1, keepdim=True) if S else size.new_zeros(H, L, 1)
        self.off = self.off + 4 * F * self.lse.unsqueeze(-1).abs().masked_fill(empty, 0.0)
        # relative error of P before it is rounded: that, exp2's (2^-21), and the sums'
        self.rel = 2 * self.off + 2.0 ** -20 + (2 * S + 64) * F

    def o_bound(self):
        u = U[self.dtype]
        # (a row's largest exponential is 1 at least where P is rounded, so that relative
        # to their sum a step is one at most)
        # (P is divided by the sum of its rounded values: with P rounded by factors 1 + d,
        # |d| <= u, o is off by sum(d P (v - o)) / (1 + sum(d P)), at most u / (1 - u)
        # sum(P |v - o|) <= u / (1 - u) (sum(P |v|) + |o|))
        return ((u / (1 - u) + self.rel) * (self.p @ self.v.abs() + self.o.abs()) + STEP[self.dtype] / 2 * self.v.abs().sum(1, keepdim=True)
                + rounding(self.o, self.dtype) + 1e-30)

    def gradients(self, do):
        """((dq, dk, dv), their bounds), each [tokens, heads, D]."""
        u, D = U[self.dtype], self.D
        do = do.double().transpose(0, 1)
        dp = do @ self.v.transpose(1, 2)
        delta = (do * self.o).sum(-1, keepdim=True)
        ds = self.p * (dp - delta)
        err = self.p * ((u + self.rel) * (dp.abs() + delta.abs()) + 2 * D * F * (do.abs() @ self.v.abs().transpose(1, 2))
                        + 2 * D * F * (do * self.o).abs().sum(-1, keepdim=True))
        # delta's own error from the output's (its rounding counts as one of P)
        err = err + self.p * (do.abs() * self.o_bound()).sum(-1, keepdim=True)
        n = 2 * (max(self.q.shape[1] * self.group, self.n) + 8) * F
        shared = lambda t: t.reshape(t.shape[0] // self.group, self.group, *t.shape[1:]).sum(1)  # noqa: E731
        dq, dk, dv = self.scale * (ds @ self.k), self.scale * (ds.transpose(1, 2) @ self.q), self.p.transpose(1, 2) @ do
        bq = self.scale * (err + n * ds.abs()) @ self.k.abs()
        bk = self.scale * (err + n * ds.abs()).transpose(1, 2) @ self.q.abs()
        bv = (self.p * (u + self.rel + n)).transpose(1, 2) @ do.abs()
        dk, dv, bk, bv = shared(dk), shared(dv), shared(bk), shared(bv)
        grads = tuple(t.transpose(0, 1) for t in (dq, dk, dv))
        bounds = tuple(t.transpose(0, 1) + rounding(g, self.dtype) + 1e-30 for t, g in zip((bq, bk, bv), grads))
        return grads, bounds


def within(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    ratio = ((got - want).abs() / bound)
    assert not torch.isnan(got).any(), (what, "NaN")
    worst = ratio.max().item() if ratio.numel() else 0.0
    assert worst <= 1.0, f"{what}: {int((ratio > 1).sum())} of {ratio.numel()} values beyond their bound, worst {worst:.3g} times it"
    return worst
