"""The operators around a block-scaled 8-bit linear layer, as measurable cases.

Each case is one pass through an operator on inputs made from a seed:

  norm      layer norm over the last dimension: a forward call, or a training
            step (forward, then the gradients of input, weight and bias).
  serve     a serving call on a weight held in 8-bit floating point with one
            scale for each 128 x 128 tile: the tokens are quantized (one scale
            for each 128 of a row) and multiplied.
  linear    one training step of the 8-bit linear layer: forward, then the
            gradients of input and weight, all three products on operands
            quantized in blocks of 128 along their own contraction.
  dropout   dropout by a counter-based generator, with or without the residual
            added in the same pass: forward and the input's gradient.
  sublayer  the three together, as a pre-norm residual branch in training:
            x + dropout(linear(norm(x))), with all gradients.

Where ``own`` is false each operator runs in its plain form: elementary torch
operations in 32 bits, rounded once at the operator's end.  ``exact`` gives
the definitions in 64 bits.

Sizes are the linears of an 8B hybrid model (hidden 4096, FFN 21504, QKV
6144, 8192 tokens) and generic odd ones; inputs follow the same distributions
as the benchmark's (Gaussian activations with sparse outliers, N(0, 0.02)
weights, small gradients with a per-row spread).
"""

import math

import numpy as np
import torch

own = False

BLOCK = 128
EPS = 1e-5
MOST = 8192 * 4096 * 21504              # T K N of the largest case
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# name: (torch type, largest finite value, exponent of its binade, mantissa bits, least normal exponent)
FORMATS = {"e4m3": (torch.float8_e4m3fn, 448.0, 8, 3, -6), "e5m2": (torch.float8_e5m2, 57344.0, 15, 2, -14)}


# ------------------------------------------------------------------ cases --
def listed():
    return [
        # decoding one sequence: the norm before a projection, all latency
        dict(name="norm_1", kind="norm", T=1, C=4096, dtype="bf16", train=False),
        # the norm of a training step at the benchmark's tokens and width
        dict(name="norm_train_8192", kind="norm", T=8192, C=4096, dtype="bf16", train=True),
        # an odd batch of an odd width, held in fp32
        dict(name="norm_train_777_odd", kind="norm", T=777, C=1357, dtype="f32", train=True),
        # decoding one sequence, the QKV projection: a weight read once
        dict(name="serve_1_qkv", kind="serve", T=1, K=4096, N=6144, scale="f32"),
        # decoding a batch of 24 sequences, the FFN up-projection
        dict(name="serve_24_ffn_up", kind="serve", T=24, K=4096, N=21504, scale="e8m0"),
        # prefill of one prompt of odd length, the FFN down-projection (long contraction)
        dict(name="serve_777_ffn_down", kind="serve", T=777, K=21504, N=4096, scale="f32"),
        # the benchmark's FFN up-projection as a training step, the largest case
        dict(name="linear_train_8192_ffn_up", kind="linear", T=8192, K=4096, N=21504, scale="e8m0", grad="e4m3"),
        # a token count and widths that are no multiples of 128, gradients of wider range
        dict(name="linear_train_1999_odd", kind="linear", T=1999, K=1360, N=3408, scale="f32", grad="e5m2"),
        # the end of a residual branch in training: dropout and the residual in one pass
        dict(name="dropout_residual_8192", kind="dropout", T=8192, C=4096, dtype="bf16", p=0.1, residual=True),
        # dropout alone on a small fp32 activation of odd width
        dict(name="dropout_300_odd", kind="dropout", T=300, C=1357, dtype="f32", p=0.25, residual=False),
        # a residual branch (attention's output projection) in training, ordinary batch
        dict(name="sublayer_2000", kind="sublayer", T=2000, C=4096, scale="e8m0", grad="e4m3", p=0.1),
        # the same on a short batch and a narrow width that is no multiple of 128
        dict(name="sublayer_333_narrow", kind="sublayer", T=333, C=1360, scale="f32", grad="e4m3", p=0.1),
    ]


def _size(rng, lo, hi):
    """Log-uniform size in [lo, hi]; half the time a multiple of 128, where
    that fits, as most model dimensions are."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and v >= 256:
        v = v // 128 * 128
    return max(lo, min(hi, v))


def draw(rng):
    kind = rng.choice(["norm", "serve", "serve", "linear", "linear", "dropout", "sublayer"])
    scale, grad = rng.choice(["f32", "e8m0"]), rng.choice(["e4m3", "e5m2"])
    if kind == "norm":
        return dict(kind=kind, T=_size(rng, 1, 8192), C=_size(rng, 64, 21504), dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    train=rng.random() < 0.7)
    if kind == "dropout":
        return dict(kind=kind, T=_size(rng, 1, 8192), C=_size(rng, 64, 21504), dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    p=round(rng.uniform(0.02, 0.6), 3), residual=rng.random() < 0.5)
    if kind == "sublayer":
        return dict(kind=kind, T=_size(rng, 64, 8192), C=_size(rng, 256, 8192), scale=scale, grad=grad,
                    p=round(rng.uniform(0.02, 0.3), 3))
    c = dict(kind=kind, T=_size(rng, 1, 4096) if kind == "serve" else _size(rng, 64, 8192), K=_size(rng, 256, 21504),
             N=_size(rng, 256, 21504), scale=scale)
    if kind == "linear":
        c["grad"] = grad
    while c["T"] * c["K"] * c["N"] > MOST // 2:
        c["K" if c["K"] >= c["N"] else "N"] //= 2
    return c


# ----------------------------------------------------------------- inputs --
def _gen(seed, role):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + role) % (1 << 62))
    return g


def _activation(seed, rows, cols, dtype=torch.bfloat16, role=0):
    g = _gen(seed, role)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    n = max(1, x.numel() // 1000)
    x.view(-1)[torch.randint(x.numel(), (n,), generator=g, device="cuda")] *= 100.0
    return x.to(dtype)


def _weight(seed, rows, cols, role=1):
    return (torch.randn(rows, cols, generator=_gen(seed, role), device="cuda") * 0.02).to(torch.bfloat16)


def _gradient(seed, rows, cols, dtype=torch.bfloat16, role=2):
    g = _gen(seed, role)
    z = torch.randn(rows, 1, generator=g, device="cuda").clamp(-3.0, 3.0)
    return (torch.randn(rows, cols, generator=g, device="cuda") * (1e-3 * torch.exp(z))).to(dtype)


def _affine(seed, C, dtype):
    g = _gen(seed, 3)
    w = 1.0 + 0.1 * torch.randn(C, generator=g, device="cuda")
    return w.to(dtype), (0.1 * torch.randn(C, generator=g, device="cuda")).to(dtype)


def prepare(case, seed):
    s = dict(case)
    kind, T = case["kind"], case["T"]
    if kind in ("norm", "dropout"):
        dtype = DTYPES[case["dtype"]]
        s["x"] = _activation(seed, T, case["C"], dtype)
        s["dy"] = _gradient(seed, T, case["C"], dtype)
        if kind == "norm":
            s["w"], s["b"] = _affine(seed, case["C"], dtype)
            if case["train"]:
                for k in ("x", "w", "b"):
                    s[k].requires_grad_()
        else:
            s["seed"], s["id"] = (int(seed) * 0x9E3779B97F4A7C15 + 1) % (1 << 63), int(seed) % 1000
            s["residual"] = _activation(seed, T, case["C"], dtype, role=4) if case["residual"] else None
            s["x"].requires_grad_()
        return s
    K, N = (case["C"], case["C"]) if kind == "sublayer" else (case["K"], case["N"])
    s["x"] = _activation(seed, T, K)
    w = _weight(seed, N, K)
    if kind == "serve":
        # what a serving program keeps of a weight: 8-bit values in rows padded to whole
        # blocks, and one scale for each 128 x 128 tile
        v, sc, code = _blocks(_pad(w.float(), 0), "e4m3", case["scale"], tiles=True)
        s["w"] = v[:N].to(torch.float8_e4m3fn).contiguous()
        s["w_scales"] = (code if case["scale"] == "e8m0" else sc).contiguous()
        return s
    s["w"] = w.requires_grad_()
    s["x"].requires_grad_()
    s["dy"] = _gradient(seed, T, N)
    if kind == "sublayer":
        s["g"], s["b"] = _affine(seed, K, torch.bfloat16)
        s["g"].requires_grad_()
        s["b"].requires_grad_()
        s["seed"], s["id"] = (int(seed) * 0x9E3779B97F4A7C15 + 1) % (1 << 63), int(seed) % 1000
    return s


# ------------------------------------------------------------ plain forms --
def _pad(x, axis):
    """Zeros up to whole blocks along both axes (0), or along the last only (1)."""
    r = 0 if axis else -x.shape[0] % BLOCK
    return torch.nn.functional.pad(x, (0, -x.shape[1] % BLOCK, 0, r))


def _power(code):
    """2^(code - 127) in fp32, for codes 1 to 254."""
    return (code.int() << 23).view(torch.float32)


def _blocks(x, fmt, scale, tiles=False):
    """The values that ``x`` (fp32, padded to whole blocks of 128 along its
    last axis, or of 128 x 128 for tiles) stands for divided by their block's
    scale, in the 8-bit format's grid; the scales, and the E8M0 codes."""
    dtype, top, top_exp, _, _ = FORMATS[fmt]
    R, C = x.shape
    v = x.view(R // BLOCK, BLOCK, C // BLOCK, BLOCK) if tiles else x.view(R, 1, C // BLOCK, BLOCK)
    a = v.abs().amax(dim=(1, 3), keepdim=True)
    if scale == "e8m0":
        m, e = torch.frexp(a)                      # a = m 2^e, m in [1/2, 1)
        e = (e - 1 - top_exp + (m > 0.875)).clamp(-126, 127)
        e = torch.where(a > 0, e, torch.zeros_like(e))
        s = _power(e + 127)
        code = (e + 127).to(torch.uint8)[:, 0, :, 0]
        y = v * (1.0 / s)
    else:
        a = torch.where(a > 0, a.clamp_min(top * 2.0 ** -126), torch.full_like(a, top))
        s, code = a / top, None
        y = v * top / a
    q = y.clamp(-top, top).to(dtype).float()
    return q.reshape(R, C), s[:, 0, :, 0], code


def _dequantized(x, fmt, scale):
    """``x`` [rows, contraction] after quantization in blocks of 128 along
    its rows, in fp32 (padded with zeros to whole blocks)."""
    q, s, _ = _blocks(_pad(x.float(), 1), fmt, scale)
    return (q.view(*s.shape, BLOCK) * s[..., None]).view(q.shape)


def _dequantized_tiles(w, scale):
    q, s, _ = _blocks(_pad(w.float(), 0), "e4m3", scale, tiles=True)
    return (q.view(s.shape[0], BLOCK, s.shape[1], BLOCK) * s[:, None, :, None]).view(q.shape)


def _words(seed, tensor_id, n):
    """One 16-bit word for each of n elements: Philox4x32-10, key the seed,
    counter (element / 8 in 64 bits, tensor id, 1)."""
    mask = 0xFFFFFFFF
    blocks = torch.arange(-(-n // 8), dtype=torch.int64, device="cuda")
    c = [blocks & mask, blocks >> 32, torch.full_like(blocks, tensor_id), torch.ones_like(blocks)]
    k0, k1 = seed & mask, seed >> 32 & mask

    def mul(m, v):
        low, high = m * (v & 0xFFFF), m * (v >> 16)
        return (high + (low >> 16)) >> 16, (low + ((high & 0xFFFF) << 16)) & mask

    for _ in range(10):
        h0, l0 = mul(0xD2511F53, c[0])
        h1, l1 = mul(0xCD9E8D57, c[2])
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    w = torch.stack(c, 1)
    return torch.stack([w & 0xFFFF, w >> 16], 2).view(-1)[:n]


def _plain_norm(x, w, b):
    x, w, b = x.float(), w.float(), b.float()
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).square().mean(1, keepdim=True) + EPS).rsqrt()
    hat = (x - mean) * rstd
    return hat * w + b, hat, rstd


def _plain_norm_grad(dy, hat, rstd, w):
    dy, g = dy.float(), dy.float() * w.float()
    dx = (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True)) * rstd
    return dx, (dy * hat).sum(0), dy.sum(0)


def _plain_keep(shape, p, seed, tensor_id):
    drop = round(p * 65536)
    keep = _words(seed, tensor_id, shape[0] * shape[1]).view(shape) >= drop
    return keep, 65536.0 / (65536 - drop)


def _plain_products(x, w, dy, fmt, scale):
    """Y, dX and dW of the 8-bit linear layer in fp32."""
    T, K = x.shape
    N = w.shape[0]
    wq = _dequantized_tiles(w, scale)
    y = _dequantized(x, "e4m3", scale) @ wq[:N].t()

    def grads(dy):
        dq = _dequantized(dy, fmt, scale)
        dx = dq @ wq[:, :K]
        dw = _dequantized(dy.t(), fmt, scale) @ _dequantized(x.t(), "e4m3", scale).t()
        return dx, dw
    return y, grads if dy is None else grads(dy)


@torch.no_grad()
def _plain(s):
    kind, x = s["kind"], s["x"]
    if kind == "norm":
        y, hat, rstd = _plain_norm(x, s["w"], s["b"])
        if not s["train"]:
            return y.to(x.dtype)
        dx, dw, db = _plain_norm_grad(s["dy"], hat, rstd, s["w"])
        return y.to(x.dtype), dx.to(x.dtype), dw.to(x.dtype), db.to(x.dtype)
    if kind == "dropout":
        keep, up = _plain_keep(x.shape, s["p"], s["seed"], s["id"])
        y = torch.where(keep, x.float() * up, torch.zeros((), device=x.device))
        dx = torch.where(keep, s["dy"].float() * up, torch.zeros((), device=x.device))
        if s["residual"] is not None:
            y = s["residual"].float() + y
        return y.to(x.dtype), dx.to(x.dtype)
    if kind == "serve":
        N, sc = s["w"].shape[0], s["w_scales"]
        if s["scale"] == "e8m0":
            sc = _power(sc)
        wq = s["w"].float() * sc.repeat_interleave(BLOCK, 0)[:N].repeat_interleave(BLOCK, 1)
        return (_dequantized(x, "e4m3", s["scale"]) @ wq.t()).to(x.dtype)
    if kind == "linear":
        y, (dx, dw) = _plain_products(x, s["w"], s["dy"], s["grad"], s["scale"])
        return y.to(x.dtype), dx.to(x.dtype), dw.to(x.dtype)
    # sublayer: each operator's result is rounded once
    h, hat, rstd = _plain_norm(x, s["g"], s["b"])
    y, grads = _plain_products(h.to(x.dtype), s["w"], None, s["grad"], s["scale"])
    keep, up = _plain_keep(y.shape, s["p"], s["seed"], s["id"])
    zero = torch.zeros((), device=x.device)
    out = x.float() + torch.where(keep, y.to(x.dtype).float() * up, zero)
    dy = torch.where(keep, s["dy"].float() * up, zero).to(x.dtype)
    dh, dw = grads(dy)
    dx, dg, db = _plain_norm_grad(dh.to(x.dtype), hat, rstd, s["g"])
    dx = dx + s["dy"].float()
    return out.to(x.dtype), dx.to(x.dtype), dg.to(x.dtype), db.to(x.dtype), dw.to(x.dtype)


# -------------------------------------------------------------------- run --
def run(state):
    s = state
    if not own:
        return _plain(s)
    import paper_2609_02846_amd as ue
    from paper_2609_02846_amd.dropout import dropout
    from paper_2609_02846_amd.fp8 import fp8_linear
    from paper_2609_02846_amd.norm import layer_norm
    from paper_2609_02846_amd.sublayer import sublayer
    kind, x = s["kind"], s["x"]
    if kind == "norm":
        y = layer_norm(x, s["w"], s["b"], EPS)
        return (y.detach(), *torch.autograd.grad(y, (x, s["w"], s["b"]), s["dy"])) if s["train"] else y
    if kind == "dropout":
        y = dropout(x, s["p"], s["seed"], s["id"], residual=s["residual"])
        return y.detach(), torch.autograd.grad(y, x, s["dy"])[0]
    if kind == "serve":
        return ue.linear_fp8(x, s["w"], s["w_scales"])
    if kind == "linear":
        y = fp8_linear(x, s["w"], scale=s["scale"], grad_fmt=s["grad"])
        return (y.detach(), *torch.autograd.grad(y, (x, s["w"]), s["dy"]))
    y = sublayer(x, s["g"], s["b"], s["w"], p=s["p"], seed=s["seed"], tensor_id=s["id"], eps=EPS, scale=s["scale"],
                 grad_fmt=s["grad"])
    return (y.detach(), *torch.autograd.grad(y, (x, s["g"], s["b"], s["w"]), s["dy"]))


# ------------------------------------------------------------------- work --
def work(case):
    kind, T = case["kind"], case["T"]
    if kind in ("norm", "dropout"):
        n, size = T * case["C"], torch.empty((), dtype=DTYPES[case["dtype"]]).element_size()
        if kind == "dropout":
            return {"bytes": size * n * (4 + bool(case["residual"])), "flops": (3 + bool(case["residual"])) * n}
        # forward: x, y, weight, bias; a step also reads dy and writes three gradients
        return {"bytes": size * ((4 if case["train"] else 2) * n + (4 if case["train"] else 2) * case["C"]),
                "flops": (20 if case["train"] else 8) * n}
    if kind == "serve":
        K, N = case["K"], case["N"]
        tiles = -(-K // BLOCK) * -(-N // BLOCK)
        return {"bytes": 2 * T * (K + N) + K * N + tiles * (1 if case["scale"] == "e8m0" else 4), "flops": 2 * T * K * N}
    K, N = (case["C"], case["C"]) if kind == "sublayer" else (case["K"], case["N"])
    # x, w and dy once; y, dx and dw once (and the norm's four vectors)
    return {"bytes": 4 * (T * K + T * N + K * N) + (8 * K if kind == "sublayer" else 0), "flops": 6 * T * K * N}


# ------------------------------------------------------------------ exact --
def _exact_quantized(x, fmt, scale, tiles=False):
    """``x`` (float64) after quantization along its rows (or in tiles), from
    the definition: each value over max / top (or over the least power of two
    from there on) goes to the nearest of the format's, ties to even; the
    scale it is held with is that power, or the fp32 number nearest to
    max / top."""
    _, top, _, bits, least = FORMATS[fmt]
    R, C = x.shape
    x = torch.nn.functional.pad(x, (0, -C % BLOCK, 0, -R % BLOCK if tiles else 0))
    h = BLOCK if tiles else 1
    v = x.reshape(x.shape[0] // h, h, x.shape[1] // BLOCK, BLOCK)
    a = v.abs().amax(3, keepdim=True).amax(1, keepdim=True)
    some = a > 0
    if scale == "e8m0":
        s = torch.exp2(torch.ceil(torch.log2(torch.where(some, a, top) / top)).clamp(-126, 127))
        y = v / s
    else:
        a = torch.where(some, a.clamp_min(top * 2.0 ** -126), top)
        s, y = (a / top).float().double(), v * top / a
    e = (torch.frexp(y)[1] - 1).clamp_min(least)
    step = torch.exp2((e - bits).double())
    q = (torch.round(y / step) * step).clamp(-top, top) * s
    return q.reshape(x.shape)[:R, :C]


def _exact_keep(case, s):
    """Philox4x32-10 in numpy's unsigned 64-bit integers."""
    n = s["x"].numel() if case["kind"] == "dropout" else case["T"] * case["C"]
    low, sixteen, half = np.uint64(0xFFFFFFFF), np.uint64(32), np.uint64(16)
    at = np.arange((n + 7) // 8, dtype=np.uint64)
    c0, c1 = at & low, at >> sixteen
    c2, c3 = np.full_like(at, s["id"]), np.full_like(at, 1)
    k0, k1 = s["seed"] % 2 ** 32, s["seed"] // 2 ** 32
    for r in range(10):
        a, b = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
        x0, x1 = np.uint64((k0 + r * 0x9E3779B9) % 2 ** 32), np.uint64((k1 + r * 0xBB67AE85) % 2 ** 32)
        c0, c1, c2, c3 = (b >> sixteen) ^ c1 ^ x0, b & low, (a >> sixteen) ^ c3 ^ x1, a & low
    w = np.empty((at.size, 8), np.uint32)
    for i, c in enumerate((c0, c1, c2, c3)):
        w[:, 2 * i], w[:, 2 * i + 1] = c & np.uint64(0xFFFF), c >> half
    t = int(np.rint(case["p"] * 65536))
    keep = torch.from_numpy(w.reshape(-1)[:n].astype(np.int64) >= t).cuda().view(case["T"], case["C"])
    return keep, 65536 / (65536 - t)


def _exact_norm(x, w, b):
    c = x - x.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt(c.pow(2).mean(1, keepdim=True) + EPS)
    return c * r * w + b


@torch.no_grad()
def exact(case, seed):
    s = prepare(case, seed)
    f64 = {k: v.detach().double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    kind, x, dy = case["kind"], f64["x"], f64.get("dy")

    def norm_grads(x, w, b, dy):
        with torch.enable_grad():
            leaves = [t.clone().requires_grad_() for t in (x, w, b)]
            return torch.autograd.grad(_exact_norm(*leaves), leaves, dy)
    if kind == "norm":
        y = _exact_norm(x, f64["w"], f64["b"])
        return (y, *norm_grads(x, f64["w"], f64["b"], dy)) if case["train"] else y
    if kind == "dropout":
        keep, up = _exact_keep(case, s)
        y = torch.where(keep, x * up, 0.0)
        return (y + f64["residual"] if case["residual"] else y), torch.where(keep, dy * up, 0.0)
    if kind == "serve":
        sc = torch.exp2(s["w_scales"].double() - 127) if case["scale"] == "e8m0" else f64["w_scales"]
        w = f64["w"] * sc.repeat_interleave(BLOCK, 0)[:case["N"]].repeat_interleave(BLOCK, 1)
        return _exact_quantized(x, "e4m3", case["scale"]) @ w[:, :case["K"]].t()

    def products(x, dy):
        wq = _exact_quantized(f64["w"], "e4m3", case["scale"], tiles=True)
        dx = _exact_quantized(dy, case["grad"], case["scale"]) @ wq
        dw = _exact_quantized(dy.t(), case["grad"], case["scale"]) @ _exact_quantized(x.t(), "e4m3", case["scale"]).t()
        return _exact_quantized(x, "e4m3", case["scale"]) @ wq.t(), dx, dw
    if kind == "linear":
        return products(x, dy)
    # what one operator hands the next is bf16, as the definition has it
    bf = lambda t: t.to(torch.bfloat16).double()  # noqa: E731
    h = bf(_exact_norm(x, f64["g"], f64["b"]))
    keep, up = _exact_keep(case, s)
    y, dh, dw = products(h, bf(torch.where(keep, dy * up, 0.0)))
    out = x + torch.where(keep, bf(y) * up, 0.0)
    dx, dg, db = norm_grads(x, f64["g"], f64["b"], bf(dh))
    return out, dx + dy, dg, db, dw
