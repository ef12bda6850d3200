"""Layer norm with more rows than the forms for few rows take: y, the
statistics and the gradients against float64 at widths on both sides of every
change of form, whole and ragged."""

import pytest
import torch

import paper_2609_02846_amd as ue
from gpu_util import say
from test_gpu_norm import ADDS, EPS, backward_check, case, check, f64, forward_ref

pytestmark = pytest.mark.gpu

# rows, columns: waves a row and vectors a lane (forward; whole or ragged)
SHAPES = [(513, 8), (520, 512), (600, 509),                          # 1 x 1
          (600, 520), (513, 1000), (600, 1001), (777, 1024),         # 1 x 2
          (600, 1032), (777, 1357), (600, 2047), (515, 2048),        # 2 x 2
          (600, 2056), (513, 3001), (600, 4095), (514, 4096),        # 4 x 2
          (513, 4104), (600, 5003), (515, 8191), (513, 8192)]        # 8 x 2
# fewer rows, for the widths whose forms do not depend on them
WIDE = [(5, 8193), (3, 12289), (7, 16383), (4, 16384), (3, 16385), (5, 20003), (4, 24575), (3, 24576), (2, 24577)]


def whole(rows, cols, dtype, ptype):
    say("norm", rows, cols, dtype, ptype)
    x, dy, w, b = case(rows, cols, dtype, ptype)
    adds = ADDS + cols // 8192 * 8
    y, mean, rstd = ue.layer_norm_forward(x, w, b, EPS, stats=True)
    X, W = f64(x), f64(w)
    Y, err, _, _, M, m_err, R, r_err = forward_ref(X, W, f64(b), adds)
    check(f64(y), Y, err, dtype, "y")
    check(f64(mean)[:, None], M, m_err, "f32", "mean")
    check(f64(rstd)[:, None], R, R * (r_err + 2.0 ** -22), "f32", "rstd")
    assert torch.equal(y, ue.layer_norm_forward(x, w, b, EPS))
    res = torch.randn(rows, cols, generator=torch.Generator().manual_seed(3)).to(x.dtype).cuda()
    dx, dw, db = ue.layer_norm_grad(x, dy, w, mean, rstd, residual_grad=res)
    backward_check(x, f64(dy), X, W, f64(mean)[:, None], f64(rstd)[:, None], dx, dw, db, f64(res), dtype, ptype, adds)


@pytest.mark.parametrize("dtype,ptype", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f32", "f32")])
def test_many_rows(dtype, ptype):
    for rows, cols in SHAPES:
        whole(rows, cols, dtype, ptype)


@pytest.mark.parametrize("dtype,ptype", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f32")])
def test_wide_rows(dtype, ptype):
    for rows, cols in WIDE:
        whole(rows, cols, dtype, ptype)


def test_rows_do_not_depend_on_how_many_there_are():
    """Forms for few and for many rows add a row's elements in another order:
    equal up to the sums' rounding, and each the same from call to call."""
    for cols in (1000, 2001, 4096):
        x, _, w, b = case(600, cols, "f32", "f32")
        y = ue.layer_norm_forward(x, w, b, EPS)
        few = ue.layer_norm_forward(x[:5].contiguous(), w, b, EPS)
        X, W, B = f64(x[:5]), f64(w), f64(b)
        Y, err, *_ = forward_ref(X, W, B, ADDS)
        check(f64(few), Y, err, "f32", "few")
        check(f64(y[:5]), Y, err, "f32", "many")
        assert torch.equal(y, ue.layer_norm_forward(x, w, b, EPS))
