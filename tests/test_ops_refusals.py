"""Refusals of the operators around the linear layers: the C entry points
return their status before anything is enqueued, and the binding raises (no
GPU is needed)."""

import ctypes
import os

import pytest
import torch

import paper_2609_02846_amd as ue
from paper_2609_02846_amd import build as ue_build
from paper_2609_02846_amd.dropout import Dropout
from paper_2609_02846_amd.fp8 import Fp8Linear, fp8_linear
from paper_2609_02846_amd.operators import COL128T, ROW128, TILE128
from paper_2609_02846_amd.sublayer import sublayer

OK, EINVAL, ESHAPE, EALIGN, ELAYOUT = ue.UE5M3_OK, ue.UE5M3_EINVAL, ue.UE5M3_ESHAPE, ue.UE5M3_EALIGN, ue.UE5M3_ELAYOUT
PTR = ctypes.c_void_p(0x100000)           # aligned, never dereferenced
ODD = ctypes.c_void_p(0x100001)
HALF = ctypes.c_void_p(0x100002)          # aligned for 16-bit elements only
BF16, F16, F32 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ue.LIB_PATH):
        ue_build.build(verbose=False)
    return ue.load_library()


def test_layer_norm(lib):
    def call(x=PTR, rows=0, cols=8, xt=BF16, w=PTR, b=PTR, pt=BF16, eps=1e-5, y=PTR, mean=None, rstd=None):
        return lib.ue5m3_layer_norm(x, rows, cols, xt, w, b, pt, eps, y, mean, rstd, None)
    assert call() == OK and call(rows=3, cols=0, x=None, y=None) == OK
    assert call(xt=3) == EINVAL and call(xt=-1) == EINVAL
    assert call(xt=BF16, pt=F16) == EINVAL and call(xt=F32, pt=BF16) == EINVAL and call(xt=F16, pt=F32) == OK
    for eps in (-1e-5, float("nan"), float("inf")):
        assert call(eps=eps) == EINVAL
    assert call(rows=-1) == ESHAPE and call(cols=-1) == ESHAPE and call(cols=2 ** 31) == ESHAPE
    assert call(rows=1, x=None) == EINVAL and call(rows=1, y=None) == EINVAL
    assert call(rows=1, x=ODD) == EALIGN and call(rows=1, w=ODD) == EALIGN and call(rows=1, mean=HALF) == EALIGN
    assert call(rows=1, pt=F32, b=HALF) == EALIGN and call(rows=1, xt=F32, pt=F32, y=HALF) == EALIGN


def test_layer_norm_grad(lib):
    def call(x=PTR, dy=PTR, rows=1, cols=8, xt=BF16, w=PTR, pt=BF16, mean=PTR, rstd=PTR, res=None, dx=PTR, dw=None,
             db=None):
        return lib.ue5m3_layer_norm_grad(x, dy, rows, cols, xt, w, pt, mean, rstd, res, dx, dw, db, None)
    assert call(rows=0) == OK and call(cols=0) == OK and call(dx=None) == OK
    assert call(xt=9) == EINVAL and call(pt=F16) == EINVAL
    assert call(rows=-2) == ESHAPE
    assert call(x=None) == EINVAL and call(dy=None) == EINVAL and call(mean=None) == EINVAL
    assert call(dx=ODD) == EALIGN and call(res=ODD) == EALIGN and call(dw=ODD) == EALIGN and call(rstd=HALF) == EALIGN


def test_dropout(lib):
    def call(x=PTR, n=0, t=BF16, p=0.5, y=PTR, res=None):
        return lib.ue5m3_dropout(x, n, t, p, 1, 2, res, y, None)
    assert call() == OK and call(p=0.0) == OK and call(p=1.0) == OK
    for p in (-0.01, 1.01, float("nan"), float("inf")):
        assert call(p=p) == EINVAL
    assert call(t=3) == EINVAL and call(n=-1) == ESHAPE and call(n=1, x=None) == EINVAL and call(n=1, y=None) == EINVAL
    assert call(n=1, x=ODD) == EALIGN and call(n=1, t=F32, res=HALF) == EALIGN


def test_quantizers(lib):
    def call(rows=0, cols=8, t=BF16, fmt=0, kind=0, x=PTR, pr=PTR, sr=PTR, pc=None, sc=None):
        return lib.ue5m3_quantize_fp8(x, rows, cols, t, fmt, kind, pr, sr, pc, sc, None)
    assert call() == OK and call(rows=4, cols=0) == OK
    assert call(t=4) == EINVAL and call(fmt=2) == EINVAL and call(kind=2) == EINVAL
    assert call(rows=-1) == ESHAPE and call(rows=2 ** 31, cols=2 ** 31) == ESHAPE
    assert call(sr=None) == EINVAL and call(pc=PTR) == EINVAL           # a pair is whole or absent
    assert call(rows=1, pr=None, sr=None) == EINVAL and call(rows=1, x=None) == EINVAL
    assert call(rows=1, x=ODD) == EALIGN and call(rows=1, pr=HALF) == EALIGN and call(rows=1, sr=HALF) == EALIGN

    def tiles(rows=0, cols=8, t=BF16, kind=0, w=PTR, p=PTR, s=PTR, pt=None, st=None):
        return lib.ue5m3_quantize_fp8_tiles(w, rows, cols, t, kind, p, s, pt, st, None)
    assert tiles() == OK and tiles(t=3) == EINVAL and tiles(kind=-1) == EINVAL and tiles(pt=PTR) == EINVAL
    assert tiles(cols=-1) == ESHAPE and tiles(rows=1, s=None) == EINVAL and tiles(rows=1, pt=HALF, st=PTR) == EALIGN


def test_gemm(lib):
    good = {0: (ROW128, {ROW128, TILE128}), 1: (ROW128, {COL128T, TILE128}), 2: (COL128T, {COL128T, TILE128})}

    def call(lay=0, M=0, N=8, K=8, a=PTR, ab=None, af=0, b=PTR, bb=TILE128, kind=0, c=PTR, ct=0, sa=PTR):
        ab = good.get(lay, (ROW128,))[0] if ab is None else ab
        return lib.ue5m3_gemm_fp8(lay, M, N, K, a, sa, ab, af, b, PTR, bb, kind, c, ct, None)
    for lay in (0, 1, 2):
        for ab in (ROW128, COL128T, TILE128):
            for bb in (ROW128, COL128T, TILE128):
                assert call(lay, ab=ab, bb=bb) == (OK if ab == good[lay][0] and bb in good[lay][1] else ELAYOUT)
    assert call(3) == ELAYOUT
    for bad in (0, 1, 2, 3, 4, 5, 9, -1):
        assert call(ab=bad) == EINVAL and call(bb=bad) == EINVAL
    assert call(af=2) == EINVAL and call(kind=2) == EINVAL and call(ct=2) == EINVAL
    assert call(M=-1) == ESHAPE and call(K=-1) == ESHAPE and call(K=2 ** 22 + 1) == ESHAPE
    assert call(M=2 ** 40, N=2 ** 40) == ESHAPE
    assert call(M=1, c=None) == EINVAL and call(M=1, a=None) == EINVAL and call(M=1, sa=None) == EINVAL
    assert call(M=1, a=HALF) == EALIGN and call(M=1, c=HALF) == EALIGN

    def serve(T=0, K=8, N=8, x=PTR, w=PTR, s=PTR, kind=0, y=PTR, yt=1):
        return lib.ue5m3_linear_fp8(x, T, K, N, w, s, kind, y, yt, None)
    assert serve() == OK and serve(kind=5) == EINVAL and serve(yt=7) == EINVAL and serve(T=-1) == ESHAPE
    assert serve(K=2 ** 22 + 1) == ESHAPE and serve(T=1, x=None) == EINVAL and serve(T=1, y=None) == EINVAL
    assert serve(T=1, x=ODD) == EALIGN and serve(T=1, w=HALF) == EALIGN and serve(T=1, y=HALF) == EALIGN
    # blocks of 128 are not blockings of the FP4 products
    for bad in (ROW128, COL128T, TILE128):
        assert lib.ue5m3_gemm(0, 0, 16, 16, PTR, PTR, bad, PTR, PTR, PTR, 2, PTR, PTR, 0, None) == EINVAL


def test_binding_refuses():
    """Host tensors, wrong types and wrong formats raise before the library is called."""
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    for f in (lambda: ue.layer_norm_forward(x), lambda: ue.dropout_forward(x, 0.1, 0), lambda: ue.quantize_fp8(x, 1),
              lambda: ue.quantize_fp8_dual(x), lambda: ue.quantize_fp8_tiles(x),
              lambda: ue.linear_fp8(x, x, x), lambda: fp8_linear(x, x.clone(), scale="f64"),
              lambda: fp8_linear(x, x.clone(), grad_fmt="e3m4"), lambda: fp8_linear(x.float(), x.clone()),
              lambda: fp8_linear(x[:, :4], x.clone()), lambda: sublayer(x, None, None, x.clone()),
              lambda: Dropout(1.5), lambda: Fp8Linear(8, 8, scale="f16", device="cpu")):
        with pytest.raises(ValueError):
            f()
