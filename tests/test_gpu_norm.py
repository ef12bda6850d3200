"""Layer norm forward and backward on the GPU against float64, with bounds
derived from the formulas."""

import numpy as np
import pytest
import torch

import paper_2609_02846_amd as ue
from gpu_util import say
from paper_2609_02846_amd.norm import LayerNorm, layer_norm

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# half a unit in the last place, relative, and the absolute floor of the type
ROUND = {"bf16": (2.0 ** -8, 1e-40), "f16": (2.0 ** -11, 2.0 ** -25), "f32": (2.0 ** -24, 1e-45)}
# additions that one of a row's sums passes through: at most 8 x 4 a lane (or,
# for the longest rows, a few hundred), 6 across the lanes, 16 waves
ADDS = 64
EPS = 1e-5


def case(rows, cols, dtype, ptype, seed=0, affine=True):
    g = torch.Generator().manual_seed(seed * 7919 + rows * 31 + cols)
    x = torch.randn(rows, cols, generator=g) * 2 + 0.5
    if cols > 4:
        x[:, cols // 3] *= 50
    dy = torch.randn(rows, cols, generator=g)
    w, b = 1 + 0.2 * torch.randn(cols, generator=g), 0.3 * torch.randn(cols, generator=g)
    t, p = TYPES[dtype], TYPES[ptype]
    return (x.to(t).cuda(), dy.to(t).cuda(), *((w.to(p).cuda(), b.to(p).cuda()) if affine else (None, None)))


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def forward_ref(x, w, b, adds):
    """y, its error bound before the output's rounding, h and h's bound."""
    u = 2.0 ** -24
    mean = x.mean(1, keepdims=True)
    d = x - mean
    var = (d * d).mean(1, keepdims=True)
    rstd = 1 / np.sqrt(var + EPS)
    mean_err = adds * u * np.abs(x).mean(1, keepdims=True)
    # the squared distances' sum: their own error, the mean's (second order and
    # its product with the distances' rounding), then square root and quotient
    rel = (adds + 8) * u + (mean_err ** 2 + 2 * mean_err * u * np.abs(d).max(1, keepdims=True)) / (var + EPS)
    h = d * rstd
    h_err = rstd * (mean_err + u * np.abs(d)) + np.abs(h) * (rel + 2 * u)
    W, B = (1.0 if w is None else w), (0.0 if b is None else b)
    y = h * W + B
    return y, np.abs(W) * h_err + 2 * u * (np.abs(h * W) + np.abs(B)), h, h_err, mean, mean_err, rstd, rel


def check(got, want, err, dtype, what):
    rel, floor = ROUND[dtype]
    bound = err + (np.abs(want) + err) * rel + floor
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} beyond the bound, worst {np.nanmax(np.abs(got - want) / bound):.3g}"


SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 8), (4, 64), (2, 509), (17, 512), (9, 513), (33, 1000), (6, 1024), (7, 1025),
          (5, 2047), (4, 2049), (300, 1357), (3, 4099), (6, 5000), (2, 8192), (3, 8200), (2, 16384), (3, 21504),
          (2, 24576), (2, 24577), (1, 40000), (1000, 96)]


@pytest.mark.parametrize("dtype,ptype", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")])
def test_forward_and_backward(dtype, ptype):
    for rows, cols in SHAPES:
        say("norm", dtype, ptype, rows, cols)
        x, dy, w, b = case(rows, cols, dtype, ptype)
        adds = ADDS + cols // 8192 * 8
        y, mean, rstd = ue.layer_norm_forward(x, w, b, EPS, stats=True)
        X, D, W, B = f64(x), f64(dy), f64(w), f64(b)
        Y, err, H, _, M, m_err, R, r_err = forward_ref(X, W, B, adds)
        check(f64(y), Y, err, dtype, "y")
        check(f64(mean)[:, None], M, m_err, "f32", "mean")
        check(f64(rstd)[:, None], R, R * (r_err + 2.0 ** -22), "f32", "rstd")
        # the backward pass takes those statistics: its own errors only
        dx, dw, db = ue.layer_norm_grad(x, dy, w, mean, rstd)
        backward_check(x, D, X, W, f64(mean)[:, None], f64(rstd)[:, None], dx, dw, db, None, dtype, ptype, adds)


def backward_check(x, D, X, W, M, R, dx, dw, db, res, dtype, ptype, adds):
    u = 2.0 ** -24
    rows, cols = X.shape
    h = (X - M) * R
    h_err = 2 * u * np.abs(h)
    g = D * W
    s1, s2 = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
    s1_err = (adds + 2) * u * np.abs(g).mean(1, keepdims=True)
    s2_err = (adds + 5) * u * np.abs(g * h).mean(1, keepdims=True)
    want = R * (g - s1 - h * s2)
    err = R * (u * np.abs(g) + s1_err + np.abs(h) * s2_err + h_err * np.abs(s2) + 4 * u * (np.abs(g) + np.abs(s1) + np.abs(h * s2)))
    if res is not None:
        want = want + res
        err = err + u * np.abs(want)
    check(f64(dx), want, err, dtype, "dx")
    n = rows / 256 + 64                               # additions of a column: a workgroup's rows, then 256 partials
    check(f64(dw), (D * h).sum(0), (n + 4) * u * np.abs(D * h).sum(0), ptype, "dweight")
    check(f64(db), D.sum(0), n * u * np.abs(D).sum(0), ptype, "dbias")


def test_many_rows_and_residual():
    for rows, cols, dtype in [(5000, 257, "f32"), (2500, 4096, "bf16"), (700, 6000, "bf16"), (600, 25000, "bf16"), (300, 9000, "f32")]:
        say("norm rows", rows, cols, dtype)
        x, dy, w, b = case(rows, cols, dtype, dtype)
        res = torch.randn(rows, cols, generator=torch.Generator().manual_seed(3)).to(x.dtype).cuda()
        _, mean, rstd = ue.layer_norm_forward(x, w, b, EPS, stats=True)
        dx, dw, db = ue.layer_norm_grad(x, dy, w, mean, rstd, residual_grad=res)
        backward_check(x, f64(dy), f64(x), f64(w), f64(mean)[:, None], f64(rstd)[:, None], dx, dw, db, f64(res), dtype,
                       dtype, ADDS + cols // 8192 * 8)
        again = ue.layer_norm_grad(x, dy, w, mean, rstd, residual_grad=res)
        for p, q in zip((dx, dw, db), again):         # fixed order of the sums
            assert torch.equal(p, q)
        only = ue.layer_norm_grad(x, dy, w, mean, rstd, need=(False, True, False))
        assert only[0] is None and only[2] is None and torch.equal(only[1], dw)
        only = ue.layer_norm_grad(x, dy, w, mean, rstd, residual_grad=res, need=(True, False, False))
        assert torch.equal(only[0], dx) and only[1] is None


def test_gradient_against_differences():
    """Central differences of the float64 forward, in random directions of x,
    weight and bias, against the kernel's gradients."""
    for rows, cols in [(3, 5), (4, 130), (2, 1500)]:
        say("norm differences", rows, cols)
        x, dy, w, b = case(rows, cols, "f32", "f32", seed=2)
        for t in (x, w, b):
            t.requires_grad_()
        grads = torch.autograd.grad(layer_norm(x, w, b, EPS), (x, w, b), dy)
        args, D = [f64(t) for t in (x, w, b)], f64(dy)
        rng, step = np.random.default_rng(5), 1e-5
        for k in range(3):
            v = rng.standard_normal(args[k].shape)
            side = [forward_ref(*[a + s * v if i == k else a for i, a in enumerate(args)], ADDS)[0] for s in (step, -step)]
            fd = ((side[0] - side[1]) * D).sum() / (2 * step)
            got = (f64(grads[k]) * v).sum()
            # binary32 gradients: about 64 units in the last place of each term
            # and 1e-7 for the differences' truncation
            assert abs(fd - got) <= 2.0 ** -17 * np.abs(f64(grads[k]) * v).sum() + 1e-6 * np.abs(D).sum(), (rows, cols, k)


def test_absent_parameters_and_empty_tensors():
    x, dy, w, b = case(5, 100, "bf16", "bf16")
    y = ue.layer_norm_forward(x)
    one, zero = torch.ones_like(w), torch.zeros_like(b)
    assert torch.equal(y, ue.layer_norm_forward(x, one, zero))
    assert torch.equal(ue.layer_norm_forward(x, w), ue.layer_norm_forward(x, w, zero))
    _, mean, rstd = ue.layer_norm_forward(x, stats=True)
    for p, q in zip(ue.layer_norm_grad(x, dy, None, mean, rstd), ue.layer_norm_grad(x, dy, one, mean, rstd)):
        assert torch.equal(p, q)
    e = torch.empty(0, 100, dtype=torch.bfloat16, device="cuda")
    y, mean, rstd = ue.layer_norm_forward(e, w, b, stats=True)
    assert y.shape == (0, 100)
    dx, dw, db = ue.layer_norm_grad(e, e, w, mean, rstd)
    assert dx.shape == (0, 100) and not dw.any() and not db.any()
    e = torch.empty(3, 0, dtype=torch.bfloat16, device="cuda")
    assert ue.layer_norm_forward(e).shape == (3, 0)


def test_special_rows():
    """A constant row gives the bias; a NaN or an infinity stays in its row."""
    x, dy, w, b = case(6, 300, "f32", "f32")
    x[1] = 3.25
    x[2, 7] = float("nan")
    x[3, 9] = float("inf")
    y, mean, rstd = ue.layer_norm_forward(x, w, b, EPS, stats=True)
    assert torch.equal(y[1], b) and torch.isnan(y[2]).all() and torch.isnan(y[3]).all()
    keep = [0, 4, 5]
    assert torch.equal(y[keep], ue.layer_norm_forward(x[keep].contiguous(), w, b, EPS))
    dx, dw, db = ue.layer_norm_grad(x, dy, w, mean, rstd)
    assert torch.isfinite(dx[[0, 1, 4, 5]]).all() and torch.isnan(dx[2]).all() and torch.isfinite(db).all()


def test_unaligned_views():
    """Tensors that start anywhere: the same bits as from aligned ones."""
    x, dy, w, b = case(7, 333, "bf16", "bf16")
    flat = torch.zeros(7 * 333 + 1, dtype=torch.bfloat16, device="cuda")
    wide = torch.zeros(334, dtype=torch.bfloat16, device="cuda")
    flat[1:] = x.view(-1)
    wide[1:] = w
    xo, wo = flat[1:].view(7, 333), wide[1:]
    assert xo.data_ptr() % 16 == 2
    y, mean, rstd = ue.layer_norm_forward(x, w, b, stats=True)
    assert torch.equal(y, ue.layer_norm_forward(xo, wo, b))
    for p, q in zip(ue.layer_norm_grad(x, dy, w, mean, rstd), ue.layer_norm_grad(xo, dy, wo, mean, rstd)):
        assert torch.equal(p, q)


def test_module_and_streams():
    torch.manual_seed(0)
    layer = LayerNorm(520)
    x = torch.randn(4, 9, 520, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    y = layer(x.transpose(0, 1))
    assert y.shape == (9, 4, 520)
    y.sum().backward()
    assert x.grad.shape == x.shape and layer.weight.grad is not None and layer.bias.grad is not None
    want = ue.layer_norm_forward(x.detach().transpose(0, 1).contiguous(), layer.weight.detach(), layer.bias.detach())
    assert torch.equal(y.detach(), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    xc = x.detach().transpose(0, 1).contiguous()
    other = ue.layer_norm_forward(xc, layer.weight.detach(), layer.bias.detach(), stream=s)
    s.synchronize()
    assert torch.equal(other, want)


def test_offsets_past_32_bits():
    """More than 2^31 elements: rows on both sides of that offset."""
    rows, cols = 2 ** 31 // 4096 + 40, 4096
    say("norm large", rows, cols)
    x = torch.randint(-8, 8, (rows, cols), dtype=torch.int8, device="cuda").to(torch.bfloat16)
    w = torch.linspace(0.5, 1.5, cols, device="cuda").to(torch.bfloat16)
    y, mean, rstd = ue.layer_norm_forward(x, w, stats=True)
    at = torch.tensor([0, 1, 2 ** 31 // cols - 1, 2 ** 31 // cols, rows - 1], device="cuda")
    assert torch.equal(y[at], ue.layer_norm_forward(x[at].contiguous(), w))
    dx, dw, _ = ue.layer_norm_grad(x, y, w, mean, rstd)
    m, r = mean[at].contiguous(), rstd[at].contiguous()
    assert torch.equal(dx[at], ue.layer_norm_grad(x[at].contiguous(), y[at].contiguous(), w, m, r)[0])
    assert torch.isfinite(dw).all()
