"""The 8-bit linear layer's parts on the GPU: quantizers byte for byte with
the oracle, products against float64, the layer's gradients, serving, graphs."""

import numpy as np
import pytest
import torch

import paper_2609_02846_amd as ue
from fp8_model import products
from gpu_util import say
from oracle import fp8 as of
from paper_2609_02846_amd.fp8 import Fp8Linear, fp8_linear
from paper_2609_02846_amd.operators import FP8, SCALE, pad128, scale_pitch

pytestmark = pytest.mark.gpu


def tensor(rows, cols, seed, dtype=torch.bfloat16, spread=2.0):
    """Normal values under a per-row and a per-column lognormal factor: block
    maxima over many binades."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(spread * torch.randn(rows, 1, generator=g))
    return (x * torch.exp(torch.randn(1, cols, generator=g))).to(dtype).cuda()


def codes(p):
    return p.view(torch.uint8).cpu().numpy()


def scales(s, n=None):
    s = s.cpu().numpy()
    v = np.exp2(s.astype(np.float64) - 127) if s.dtype == np.uint8 else s.astype(np.float64)
    return v if n is None else v[:, :n]


def same(got, want, fmt):
    """Codes equal, any NaN code for a NaN."""
    g, w = of.decode(got, fmt), of.decode(want, fmt)
    nan = np.isnan(w)
    assert np.array_equal(np.isnan(g), nan)
    assert np.array_equal(got[~nan], want[~nan])


SHAPES = [(1, 1), (1, 128), (2, 129), (127, 8), (128, 128), (130, 260), (77, 1357), (300, 511), (513, 40)]


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_rows_and_columns(dtype, fmt, scale):
    for R, C in SHAPES:
        say("quantize", dtype, fmt, scale, R, C)
        x = tensor(R, C, R + C, dtype, 0.5 if dtype == torch.float16 else 2.0)
        X = x.double().cpu().numpy()
        (pr, sr), (pc, sc) = ue.quantize_fp8_dual(x, fmt, scale)
        assert pr.shape == (R, pad128(C)) and pc.shape == (C, pad128(R)) and pr.dtype == FP8[fmt]
        assert sr.shape == (pad128(C) // 128, scale_pitch(R)) and sr.dtype == SCALE[scale]
        for p, s, src in ((pr, sr, X), (pc, sc, X.T)):
            q, w = of.quantize_rows(src, fmt, scale)
            same(codes(p), q, fmt)
            assert np.array_equal(scales(s, src.shape[0]), w)
        for axis, (p, s) in ((1, (pr, sr)), (0, (pc, sc))):
            p1, s1 = ue.quantize_fp8(x, axis, fmt, scale)
            n = C if axis == 0 else R
            assert np.array_equal(codes(p1), codes(p)) and torch.equal(s1[:, :n], s[:, :n])


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
def test_tiles(scale):
    for R, C in SHAPES + [(260, 700)]:
        say("tiles", scale, R, C)
        w = tensor(R, C, 3 * R + C)
        p, s, pt, st = ue.quantize_fp8_tiles(w, scale)
        q, sw = of.quantize_tiles(w.double().cpu().numpy(), scale)
        assert np.array_equal(codes(p), q) and np.array_equal(scales(s), sw)
        assert torch.equal(st, s.t()) and pt.shape == (C, pad128(R))
        assert np.array_equal(codes(pt)[:, :R], q[:, :C].T) and not codes(pt)[:, R:].any()
        p1, s1, none, _ = ue.quantize_fp8_tiles(w, scale, transposed=False)
        assert none is None and np.array_equal(codes(p1), q) and torch.equal(s1, s)


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_every_bf16_value(fmt, scale):
    """All 65536 bit patterns, each block holding one binade and its neighbours
    (the extremes of the range among them), with NaN and infinities."""
    bits = np.arange(65536, dtype=np.uint16).reshape(512, 128)
    x = torch.from_numpy(bits.view(np.int16).copy()).view(torch.bfloat16).cuda()
    X = x.double().cpu().numpy()
    p, s = ue.quantize_fp8(x, 1, fmt, scale)
    q, w = of.quantize_rows(X, fmt, scale)
    same(codes(p), q, fmt)
    assert np.array_equal(scales(s, 512), w)
    mixed = x[torch.randperm(512, generator=torch.Generator().manual_seed(1)).cuda()].contiguous()
    p, s = ue.quantize_fp8(mixed, 0, fmt, scale)
    q, w = of.quantize_rows(mixed.double().cpu().numpy().T, fmt, scale)
    same(codes(p), q, fmt)
    assert np.array_equal(scales(s, 128), w)


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
def test_fp32_inputs(scale):
    """binary32 elements: the quotient may be rounded twice, so a code may be
    the neighbour where the exact quotient lies within 2^-22 of a midpoint."""
    x = tensor(90, 300, 5, torch.float32)
    p, s = ue.quantize_fp8(x, 1, "e4m3", scale)
    X = x.double().cpu().numpy()
    q, w = of.quantize_rows(X, "e4m3", scale)
    got = codes(p)
    assert np.array_equal(scales(s, 90), w)
    off = got != q
    if scale == "e8m0":
        assert not off.any()                          # division by a power of two
    d = np.abs(of.decode(got, "e4m3") - of.decode(q, "e4m3"))[off]
    y = np.abs(np.pad(X, ((0, 0), (0, 84))) / np.repeat(w.T, 128, 1))[off]
    mid = (np.abs(of.decode(got, "e4m3")) + np.abs(of.decode(q, "e4m3")))[off] / 2
    assert (np.abs(y - mid) <= 2.0 ** -22 * mid).all() and d.size <= 4


def operands(M, N, K, scale, a_fmt, tiled, seed):
    """Random finite codes and scales (not a quantizer's: every code, scales
    over ten binades), and their float64 values."""
    rng = np.random.default_rng(seed)

    def payload(rows, fmt):
        c = rng.integers(0, 256, (rows, pad128(K)), dtype=np.uint8)
        c = np.where(np.isnan(of.decode(c, fmt)), 0x31, c).astype(np.uint8)
        if fmt == "e5m2":                             # keep the products of one order
            c = np.where((c & 0x7F) > 0x50, c & 0xBF, c).astype(np.uint8)
        c[:, K:] = 0
        return c

    def scale_array(shape):
        if scale == "e8m0":
            return rng.integers(120, 130, shape, dtype=np.uint8)
        return (2.0 ** rng.uniform(-7, 3, shape)).astype(np.float32)
    kb = pad128(K) // 128
    a, b = payload(M, a_fmt), payload(N, "e4m3")
    sa, sb = scale_array((kb, scale_pitch(M))), scale_array((pad128(N) // 128, kb) if tiled else (kb, scale_pitch(N)))
    value = lambda s: np.exp2(s.astype(np.float64) - 127) if scale == "e8m0" else s.astype(np.float64)  # noqa: E731
    A = held(a, value(sa)[:, :M], a_fmt)
    B = held(b, np.repeat(value(sb), 128, 0)[:N].T if tiled else value(sb)[:, :N], "e4m3")
    up = lambda v: torch.from_numpy(v).cuda()  # noqa: E731
    return up(a).view(FP8[a_fmt]), up(sa), up(b).view(FP8["e4m3"]), up(sb), A, B


def held(codes, scales, fmt):
    """An operand's values [rows, pad(K)], scales [rows, blocks] and format, from
    codes and scales [blocks, rows]."""
    return torch.from_numpy(of.decode(codes, fmt)).cuda(), torch.from_numpy(np.ascontiguousarray(scales.T)).cuda(), fmt


def quantized(x, fmt, scale):
    return held(*of.quantize_rows(x, fmt, scale), fmt)


def quantized_tiles(w, scale, transposed=False):
    q, s = of.quantize_tiles(w, scale)
    if transposed:
        q, s = np.pad(q, ((0, -q.shape[0] % 128), (0, 0)))[:, :w.shape[1]].T, s.T
    return held(q, np.repeat(s, 128, 0)[:q.shape[0]].T, "e4m3")


def product_check(c, A, B, K, what, bf16=False):
    """binary32 accumulation of K products: |C - AB| <= K 2^-23 |A||B| (the
    recursive-sum bound with a factor of two for products of a block and
    scales), plus the output's rounding; AB as the matrix instructions define
    it."""
    want, mag = (t.cpu().numpy() for t in products(*A, *B))
    err = np.abs(c.detach().double().cpu().numpy() - want)
    bound = (K + 8) * 2.0 ** -23 * mag
    bound = bound + (np.abs(want) + bound) * (2.0 ** -8 if bf16 else 2.0 ** -23) + 1e-38
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} beyond the bound, worst {np.nanmax(err / bound):.3g}"
    norm = np.linalg.norm(want)
    # errors of many terms partly cancel: far below the bound in the norm
    assert np.linalg.norm(err) <= (2.0 ** -8 if bf16 else 2.0 ** -18) * norm + 1e-30, what


GEMMS = [(1, 1, 1), (1, 16, 128), (1, 300, 257), (3, 130, 640), (16, 64, 1000), (17, 129, 4096), (33, 500, 300),
         (64, 1000, 777), (65, 128, 129), (128, 128, 128), (129, 257, 511), (200, 96, 2000), (256, 256, 384),
         (300, 700, 1024), (513, 385, 260), (1, 4100, 3000), (24, 2050, 1111)]


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("a_fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("tiled", [False, True])
def test_products(scale, a_fmt, tiled):
    for i, (M, N, K) in enumerate(GEMMS):
        say("gemm_fp8", scale, a_fmt, tiled, M, N, K)
        a, sa, b, sb, A, B = operands(M, N, K, scale, a_fmt, tiled, i)
        blk = dict(b_blk="tile" if tiled else "row")
        guard = torch.full((M * N + 64,), 7.0, device="cuda")
        out = guard[:M * N].view(M, N)
        c = ue.gemm_fp8("nt", M, N, K, a, sa, b, sb, out=out, **blk)
        product_check(c, A, B, K, f"{M} {N} {K} fp32")
        assert (guard[M * N:] == 7.0).all()
        c = ue.gemm_fp8("nt", M, N, K, a, sa, b, sb, **blk)
        product_check(c, A, B, K, f"{M} {N} {K} bf16", True)


def test_layouts_and_empty_products():
    M, N, K = 130, 200, 300
    a, sa, b, sb, _, _ = operands(M, N, K, "f32", "e5m2", True, 9)
    want = ue.gemm_fp8("nt", M, N, K, a, sa, b, sb, out_dtype=torch.float32)
    assert torch.equal(want, ue.gemm_fp8("nn", M, N, K, a, sa, b, sb, out_dtype=torch.float32))
    a, sa, b, sb, _, _ = operands(M, N, K, "e8m0", "e4m3", False, 9)
    want = ue.gemm_fp8("nt", M, N, K, a, sa, b, sb, b_blk="row", out_dtype=torch.float32)
    assert torch.equal(want, ue.gemm_fp8("tn", M, N, K, a, sa, b, sb, out_dtype=torch.float32))
    assert not ue.gemm_fp8("nt", M, N, 0, a, sa, b, sb).any()
    assert ue.gemm_fp8("nt", 0, N, K, a, sa, b, sb).shape == (0, N)
    with pytest.raises(ue.UE5M3Error):
        ue.gemm_fp8("tn", M, N, K, a, sa, b, sb, a_blk="row")
    with pytest.raises(ValueError):
        ue.gemm_fp8("nt", M, N, K, a, sa, b, sb.float().contiguous(), b_blk="row")
    with pytest.raises(ValueError):
        ue.gemm_fp8("nt", M + 16, N, K, a, sa, b, sb, b_blk="row")


def test_integer_products_are_exact():
    """Small whole numbers under scales of one: every sum is exact."""
    rng = np.random.default_rng(3)
    for M, N, K in [(1, 128, 128), (5, 70, 256), (96, 200, 512), (300, 300, 1000)]:
        A, B = rng.integers(-8, 9, (M, K)), rng.integers(-8, 9, (N, K))
        enc = lambda v: torch.from_numpy(of.encode(np.pad(v, ((0, 0), (0, -K % 128))).astype(np.float64), "e4m3")).cuda()  # noqa: E731
        a, b, kb = enc(A).view(FP8["e4m3"]), enc(B).view(FP8["e4m3"]), pad128(K) // 128
        for kind, one in (("f32", 1.0), ("e8m0", 127)):
            full = lambda *s: torch.full(s, one, dtype=SCALE[kind], device="cuda")  # noqa: E731
            c = ue.gemm_fp8("nt", M, N, K, a, full(kb, scale_pitch(M)), b, full(pad128(N) // 128, kb), out_dtype=torch.float32)
            assert np.array_equal(c.cpu().numpy(), (A @ B.T).astype(np.float32)), (M, N, K, kind)


# enough 256 x 256 tiles for the kernel of large products (one and several a
# workgroup, ragged edges, odd and even numbers of blocks, one block)
LARGE = [(2900, 2950, 384), (4100, 4200, 520), (2816, 3330, 100), (6000, 4097, 1290)]


@pytest.mark.parametrize("tiled", [False, True])
@pytest.mark.parametrize("scale", ["f32", "e8m0"])
def test_large_products(scale, tiled):
    """Whole numbers (every output exact) under scales that are powers of two
    and differ from row to row, and sampled outputs of random codes."""
    rng = np.random.default_rng(11)
    for M, N, K in LARGE:
        say("gemm_fp8 large", scale, tiled, M, N, K)
        kb = pad128(K) // 128
        a = torch.randint(-4, 5, (M, pad128(K)), device="cuda").float()
        b = torch.randint(-4, 5, (N, pad128(K)), device="cuda").float()
        a[:, K:] = b[:, K:] = 0
        ea = torch.randint(0, 4, (kb, scale_pitch(M)), device="cuda")
        eb = torch.randint(0, 4, (pad128(N) // 128, kb) if tiled else (kb, scale_pitch(N)), device="cuda")
        enc = (lambda e: torch.exp2(e.float())) if scale == "f32" else (lambda e: (e + 127).to(torch.uint8))
        rows_b = eb.repeat_interleave(128, 0)[:N] if tiled else eb[:, :N].t()
        wide = lambda v, e: (v.view(v.shape[0], kb, 128) * torch.exp2(e.float())[:, :, None]).view(v.shape)  # noqa: E731
        want = wide(a, ea[:, :M].t()) @ wide(b, rows_b).t()      # below 2^24: exact in binary32
        for fmt in ("e4m3", "e5m2"):
            args = (a.to(FP8[fmt]), enc(ea).contiguous(), b.to(FP8["e4m3"]), enc(eb).contiguous())
            blk = "tile" if tiled else "row"
            guard = torch.full((M * N + 64,), 7.0, device="cuda")
            c = ue.gemm_fp8("nt", M, N, K, *args, b_blk=blk, out=guard[:M * N].view(M, N))
            assert torch.equal(c, want) and (guard[M * N:] == 7.0).all()
            assert torch.equal(ue.gemm_fp8("nt", M, N, K, *args, b_blk=blk), want.to(torch.bfloat16))
        ops = operands(M, N, K, scale, "e5m2", tiled, M)
        c = ue.gemm_fp8("nt", M, N, K, *ops[:4], b_blk="tile" if tiled else "row", out_dtype=torch.float32)
        m, n = (torch.from_numpy(rng.choice(v, 150, replace=False)).cuda() for v in (M, N))
        product_check(c[m][:, n], (ops[4][0][m], ops[4][1][m], ops[4][2]), (ops[5][0][n], ops[5][1][n], ops[5][2]), K,
                      f"{M} {N} {K}")


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("M,N,K,tiled", [(1, 21504, 130, True), (1, 9000, 520, False), (20, 20011, 257, True),
                                         (40, 9001, 1024, False), (64, 12345, 384, True)])
def test_few_rows_by_many_columns(M, N, K, tiled, scale):
    """Several groups of B's rows for each workgroup, and a last round that
    leaves some of them idle."""
    say("few rows", M, N, K, tiled, scale)
    a, sa, b, sb, A, B = operands(M, N, K, scale, "e4m3", tiled, N)
    c = ue.gemm_fp8("nt", M, N, K, a, sa, b, sb, b_blk="tile" if tiled else "row", out_dtype=torch.float32)
    product_check(c, A, B, K, f"{M} {N} {K}")
    if tiled and M * pad128(K) <= 8192:               # quantized where it is multiplied
        x = tensor(M, K, N)
        A = quantized(x.double().cpu().numpy(), "e4m3", scale)
        product_check(ue.linear_fp8(x, b, sb, out_dtype=torch.float32), A, B, K, f"serve {M} {N} {K}")


# more rounds of 128 rows than of 256; too few tiles of 256 rows for every CU, so split
TALL = [(1990, 2501, 300), (630, 3301, 12700)]


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("a_fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("tiled", [False, True])
def test_tall_tiles(scale, a_fmt, tiled):
    """Products of 256 x 128 tiles: every row at some columns and every column at some rows."""
    for M, N, K in TALL:
        say("tall", M, N, K, scale, a_fmt, tiled)
        a, sa, b, sb, A, B = operands(M, N, K, scale, a_fmt, tiled, M)
        blk = dict(b_blk="tile" if tiled else "row")
        guard = torch.full((M * N + 64,), 7.0, device="cuda")
        c = ue.gemm_fp8("nt", M, N, K, a, sa, b, sb, out=guard[:M * N].view(M, N), **blk)
        assert (guard[M * N:] == 7.0).all()
        half = ue.gemm_fp8("nt", M, N, K, a, sa, b, sb, **blk)
        m = torch.tensor([0, 15, 63, 64, 127, 255, 256, 300, M - 1], device="cuda")
        n = torch.tensor([0, 3, 15, 64, 127, 128, 200, N - 2, N - 1], device="cuda")
        for rows, cols in ((torch.arange(M, device="cuda"), n), (m, torch.arange(N, device="cuda"))):
            As, Bs = (A[0][rows], A[1][rows], A[2]), (B[0][cols], B[1][cols], B[2])
            product_check(c[rows][:, cols], As, Bs, K, f"{M} {N} {K} fp32")
            product_check(half[rows][:, cols], As, Bs, K, f"{M} {N} {K} bf16", True)


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
def test_bad_values_stay_in_their_row(scale):
    """A NaN token spoils its own outputs and nothing else."""
    for T in (3, 20, 140):
        x, w = tensor(T, 300, 1), tensor(260, 300, 2)
        p, s, _, _ = ue.quantize_fp8_tiles(w, scale, transposed=False)
        want = ue.linear_fp8(x, p, s)
        x[1, 17] = float("nan")
        x[2, 0] = float("inf")
        y = ue.linear_fp8(x, p, s)
        keep = [i for i in range(T) if i not in (1, 2)]
        assert torch.isnan(y[1:3]).all() and torch.equal(y[keep], want[keep])


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("T", [1, 2, 7, 16, 33, 64, 200])
def test_serving_equals_quantize_and_multiply(T, scale):
    for K, N in [(256, 128), (1000, 300), (4096, 520), (130, 1), (8000, 96)]:
        say("linear_fp8", T, K, N, scale)
        x, w = tensor(T, K, T + K), tensor(N, K, N)
        p, s, _, _ = ue.quantize_fp8_tiles(w, scale, transposed=False)
        A = quantized(x.double().cpu().numpy(), "e4m3", scale)
        B = held(codes(p), np.repeat(scales(s), 128, 0)[:N].T, "e4m3")
        product_check(ue.linear_fp8(x, p, s, out_dtype=torch.float32), A, B, K, f"serve {T} {K} {N}")
        product_check(ue.linear_fp8(x, p, s), A, B, K, f"serve {T} {K} {N} bf16", True)


@pytest.mark.parametrize("scale,grad", [("f32", "e4m3"), ("e8m0", "e4m3"), ("e8m0", "e5m2"), ("f32", "e5m2")])
def test_layer_gradients(scale, grad):
    """Y, dX and dW equal the products of the oracle's quantized operands."""
    for T, K, N in [(1, 130, 70), (100, 200, 300), (257, 384, 129)]:
        say("fp8_linear", scale, grad, T, K, N)
        x, w, dy = tensor(T, K, 1).requires_grad_(), tensor(N, K, 2, spread=0.3).requires_grad_(), tensor(T, N, 3)
        y = fp8_linear(x, w, scale, grad)
        dx, dw = torch.autograd.grad(y, (x, w), dy)
        X, W, D = (t.detach().double().cpu().numpy() for t in (x, w, dy))
        product_check(y, quantized(X, "e4m3", scale), quantized_tiles(W, scale), K, "Y", True)
        product_check(dx, quantized(D, grad, scale), quantized_tiles(W, scale, True), N, "dX", True)
        product_check(dw, quantized(D.T, grad, scale), quantized(X.T, "e4m3", scale), T, "dW", True)
        for need in ((True, False), (False, True)):
            a, b = x.detach().requires_grad_(need[0]), w.detach().requires_grad_(need[1])
            y2 = fp8_linear(a, b, scale, grad)
            g, = torch.autograd.grad(y2, a if need[0] else b, dy)
            assert torch.equal(y2, y) and torch.equal(g, dx if need[0] else dw)


def test_gradient_against_differences():
    """The layer is linear in dY's values and bilinear in X and W: where
    quantization is exact (whole numbers up to 8), a difference of the forward
    pass is the gradient."""
    rng = np.random.default_rng(1)
    # the largest of each block is a power of two, so that E8M0 blocks hold whole numbers exactly
    whole = lambda r, c: torch.from_numpy(rng.integers(-7, 8, (r, c)).astype(np.float32)).to(torch.bfloat16).cuda()  # noqa: E731
    x, w, dy = whole(40, 100).requires_grad_(), whole(60, 100).requires_grad_(), whole(40, 60)
    dx, dw = torch.autograd.grad(fp8_linear(x, w), (x, w), dy)
    f = lambda a, b: (fp8_linear(a.detach(), b.detach()).double() * dy.double()).sum().item()  # noqa: E731
    for i, j in [(0, 0), (13, 99), (39, 50)]:
        e = torch.zeros_like(x)
        e[i, j] = 1.0
        fd = (f(x + e, w) - f(x - e, w)) / 2
        # dX and each Y in bf16: sums of 60 products below 60 * 7 * 7, their
        # rounding and that of 2 x 60 outputs of up to 4900
        assert abs(fd - dx[i, j].item()) <= 60 * 7 * 4900 * 2.0 ** -9 / 2
        direct = (dy[i].double() @ w[:, j].detach().double()).item()
        assert abs(dx[i, j].item() - direct) <= abs(direct) * 2.0 ** -8
    for n, k in [(0, 0), (59, 99), (30, 20)]:
        direct = (dy[:, n].double() @ x[:, k].detach().double()).item()
        assert abs(dw[n, k].item() - direct) <= abs(direct) * 2.0 ** -8


def test_module_empty_and_frozen():
    layer = Fp8Linear(200, 130)
    x = torch.randn(2, 5, 200, device="cuda").to(torch.bfloat16)
    y = layer(x)
    assert y.shape == (2, 5, 130)
    y.float().sum().backward()
    assert layer.weight.grad.shape == (130, 200)
    with torch.no_grad():
        assert torch.equal(layer.freeze()(x), layer.unfreeze()(x))
    e = torch.empty(0, 200, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    y = layer(e)
    g = torch.autograd.grad(y, (e, layer.weight), torch.empty_like(y))
    assert y.shape == (0, 130) and g[0].shape == (0, 200) and not g[1].any()


def test_no_tokens_with_a_weight_gradient_alone():
    w = tensor(130, 200, 2).requires_grad_()
    y = fp8_linear(torch.empty(0, 200, device="cuda", dtype=torch.bfloat16), w)
    dw, = torch.autograd.grad(y, w, torch.empty_like(y))
    assert y.shape == (0, 130) and dw.shape == w.shape and not dw.any()


def test_streams_and_graph():
    """A serving call on another stream, and captured: every replay equals the
    eager result, with eager work between the replays."""
    w = tensor(700, 900, 2)
    p, s, _, _ = ue.quantize_fp8_tiles(w, "f32", transposed=False)
    for T in (1, 40, 300):
        x = tensor(T, 900, T)
        want = ue.linear_fp8(x, p, s)
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            out = ue.linear_fp8(x, p, s)
        st.synchronize()
        assert torch.equal(out, want)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            ue.linear_fp8(x, p, s, out=out)
        for i in range(3):
            out.zero_()
            ue.linear_fp8(tensor(T, 900, 50 + i), p, s)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
