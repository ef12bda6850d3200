"""Refusals of the operators between the QKV and the output projection: the C entry
points return their status before anything is enqueued, the binding raises (no GPU is
needed)."""

import ctypes
import os

import pytest
import torch

import paper_2609_02846_amd as ue
from paper_2609_02846_amd import AttentionC, AttentionGradC, PagedAttentionC, PagesC, RopeC
from paper_2609_02846_amd import build as ue_build
from paper_2609_02846_amd.attention import attention, paged_attention
from paper_2609_02846_amd.paged import PagedCache, copy_pages
from paper_2609_02846_amd.rotary import qk_norm_rope, qk_norm_rope_append, rotary_frequencies

OK, EINVAL, ESHAPE, EALIGN = ue.UE5M3_OK, ue.UE5M3_EINVAL, ue.UE5M3_ESHAPE, ue.UE5M3_EALIGN
PTR, ODD, HALF = 0x100000, 0x100001, 0x100002    # aligned, never dereferenced; for bytes, for 16 bits only
BF16, F16, F32 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ue.LIB_PATH):
        ue_build.build(verbose=False)
    return ue.load_library()


def rope_args(**kw):
    a = dict(tokens=0, q_heads=4, kv_heads=2, dim=64, pairs=32, type=BF16, weight_type=BF16, norm=1, interleaved=0,
             eps=1e-6, amplitude=1.0, q=PTR, k=PTR, q_token=256, q_head=64, k_token=128, k_head=64, q_weight=PTR, k_weight=PTR,
             positions=PTR, period=1, freqs=PTR, q_out=PTR, k_out=PTR, q_out_token=256, q_out_head=64, k_out_token=128,
             k_out_head=64)
    a.update(kw)
    return RopeC(**a)


def pages(**kw):
    a = dict(k=PTR, v=PTR, pages=10, page_size=16, page=2048, token=64, head=1024)
    a.update(kw)
    return PagesC(**a)


BAD_ROPE = [(dict(type=3), EINVAL), (dict(type=-1), EINVAL), (dict(weight_type=F16), EINVAL), (dict(type=F32), EINVAL),
            (dict(norm=2), EINVAL), (dict(interleaved=-1), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL),
            (dict(amplitude=float("inf")), EINVAL), (dict(positions=None, period=0), EINVAL), (dict(tokens=-1), ESHAPE),
            (dict(tokens=2 ** 41), ESHAPE), (dict(q_heads=-1), ESHAPE), (dict(kv_heads=-1), ESHAPE), (dict(q_heads=2 ** 17), ESHAPE),
            (dict(dim=0), ESHAPE), (dict(dim=257), ESHAPE), (dict(pairs=33), ESHAPE), (dict(pairs=-1), ESHAPE),
            (dict(tokens=1, q=None), EINVAL), (dict(tokens=1, k=None), EINVAL), (dict(tokens=1, freqs=None), EINVAL),
            (dict(tokens=1, q_out=None), EINVAL), (dict(tokens=1, q=ODD), EALIGN), (dict(tokens=1, k=ODD), EALIGN),
            (dict(tokens=1, q_out=ODD), EALIGN), (dict(tokens=1, q_weight=ODD), EALIGN), (dict(tokens=1, freqs=HALF), EALIGN),
            (dict(tokens=1, positions=0x100004), EALIGN), (dict(tokens=1, weight_type=F32, k_weight=HALF), EALIGN)]


def test_rope(lib):
    assert lib.ue5m3_qk_norm_rope(rope_args(), None) == OK and lib.ue5m3_qk_norm_rope(None, None) == EINVAL
    for kw, want in BAD_ROPE + [(dict(q_heads=0), ESHAPE), (dict(norm=0, pairs=0), EINVAL), (dict(tokens=1, k_out=None), EINVAL),
                                (dict(tokens=1, k_out=ODD), EALIGN)]:
        assert lib.ue5m3_qk_norm_rope(rope_args(**kw), None) == want, kw


def test_rope_grad(lib):
    def call(gq=PTR, gk=PTR, dqw=None, dkw=None, scratch=PTR, **kw):
        return lib.ue5m3_qk_norm_rope_grad(rope_args(**kw), gq, gk, dqw, dkw, scratch, None)
    assert call() == OK
    for kw, want in BAD_ROPE:
        if "q_out" not in kw or want == EALIGN:         # (dq is nullable)
            assert call(**kw) == want, kw
    assert call(norm=0, dqw=PTR) == EINVAL and call(dqw=ODD) == EALIGN and call(weight_type=F32, dkw=HALF) == EALIGN
    assert call(scratch=HALF) == EALIGN
    assert call(tokens=1, gq=None) == EINVAL and call(tokens=1, gk=None) == EINVAL and call(tokens=1, dqw=PTR, scratch=None) == EINVAL
    assert call(tokens=1, gq=ODD) == EALIGN and call(tokens=1, gk=ODD) == EALIGN
    n = lib.ue5m3_qk_norm_rope_grad_scratch
    assert n(0, 4, 64) == 0 and n(-1, 4, 64) == 0 and n(1, 1, 64) == 2 * 64 * 4 and n(2 ** 30, 40, 128) <= 1 << 22


def test_append(lib):
    def call(v=PTR, cache=None, slots=PTR, **kw):
        return lib.ue5m3_qk_norm_rope_append(rope_args(**kw), v, 128, 64, pages() if cache is None else cache, slots, None)
    assert call() == OK and call(q_heads=0, q=None, q_out=None, norm=0, pairs=0) == OK
    for kw, want in BAD_ROPE:
        assert call(**kw) == want, kw
    for size in (0, -1, 3, 24, -(2 ** 31)):
        assert call(cache=pages(page_size=size)) == EINVAL
    assert call(cache=pages(pages=-1)) == ESHAPE and call(cache=pages(pages=2 ** 31 + 1)) == ESHAPE and call(kv_heads=0) == ESHAPE
    assert call(tokens=1, v=None) == EINVAL and call(tokens=1, slots=None) == EINVAL and call(tokens=1, cache=pages(k=None)) == EINVAL
    assert call(tokens=1, v=ODD) == EALIGN and call(tokens=1, cache=pages(v=ODD)) == EALIGN and call(tokens=1, slots=0x100004) == EALIGN
    assert lib.ue5m3_qk_norm_rope_append(rope_args(), PTR, 128, 64, None, PTR, None) == EINVAL


def test_copy_pages(lib):
    def call(src, dst, base=PTR, planes=1, plane=1000, n_pages=10, page=100, n=None):
        s, d = ((ctypes.c_int32 * max(len(x), 1))(*x) for x in (src, dst))
        return lib.ue5m3_copy_pages(base, planes, plane, n_pages, page, s, d, len(src) if n is None else n, None)
    assert call([], []) == OK and call([1], [2], planes=0) == OK and call([1], [2], page=0) == OK
    for src, dst in [([1], [1]), ([1, 2], [3, 3]), ([1, 2], [2, 3]), ([1, 2], [3, 1]), ([-1], [2]), ([1], [-1]), ([10], [1]), ([1], [10]),
                     ([0], [2 ** 31 - 1])]:
        assert call(src, dst) == EINVAL, (src, dst)
    assert call([1, 1], [2, 3], base=None) == EINVAL
    assert call([1], [2], n=-1) == ESHAPE and call([1], [2], n=11) == ESHAPE and call([1], [2], planes=-1) == ESHAPE
    assert call([1], [2], page=101) == ESHAPE and call([1], [2], plane=1001) == ESHAPE and call([1], [2], planes=2, plane=998) == ESHAPE
    assert call([1], [2], n_pages=2 ** 31, page=2 ** 40) == ESHAPE and call([1], [2], base=ODD) == EALIGN
    assert lib.ue5m3_copy_pages(PTR, 1, 1000, 10, 100, None, None, 1, None) == EINVAL


def attention_args(**kw):
    a = dict(q_tokens=0, k_tokens=0, sequences=1, q_starts=PTR, k_starts=PTR, q_heads=4, kv_heads=2, dim=64, type=BF16, causal=1,
             scale=0.1, window=0, sinks=0, q=PTR, k=PTR, v=PTR, q_token=256, q_head=64, k_token=128, k_head=64, v_token=128,
             v_head=64, o=PTR, o_rest=PTR, lse=PTR)
    a.update(kw)
    return AttentionC(**a)


BAD_HEADS = [(dict(type=F32), EINVAL), (dict(type=7), EINVAL), (dict(scale=0.0), EINVAL), (dict(scale=-1.0), EINVAL),
             (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(q_heads=3), ESHAPE), (dict(q_heads=0), ESHAPE),
             (dict(kv_heads=0), ESHAPE), (dict(dim=0), ESHAPE), (dict(dim=136), ESHAPE), (dict(dim=60), ESHAPE),
             (dict(window=-1), ESHAPE), (dict(sinks=-1), ESHAPE)]
BAD_ATTENTION = BAD_HEADS + [
    (dict(causal=2), EINVAL), (dict(causal=0, window=5), EINVAL), (dict(q_starts=None), EINVAL), (dict(k_starts=None), EINVAL),
    (dict(q_tokens=-1), ESHAPE), (dict(k_tokens=-1), ESHAPE), (dict(q_tokens=2 ** 30 + 1), ESHAPE), (dict(sequences=0), ESHAPE),
    (dict(q_tokens=5, k_tokens=4, sequences=2, q_starts=None, k_starts=None), ESHAPE), (dict(q_tokens=2, q_token=56), ESHAPE),
    (dict(q_tokens=2, q_token=2 ** 23), ESHAPE), (dict(q_head=8), ESHAPE), (dict(k_tokens=2, k_token=0), ESHAPE),
    (dict(k_tokens=2, v_token=-128), ESHAPE), (dict(q_tokens=2 ** 30, q_heads=2 ** 16), ESHAPE), (dict(sequences=2 ** 30), ESHAPE),
    (dict(q_tokens=1, q=None), EINVAL), (dict(q_tokens=1, o=None), EINVAL), (dict(k_tokens=1, k=None), EINVAL),
    (dict(k_tokens=1, v=None), EINVAL), (dict(q=0x100008), EALIGN), (dict(k=HALF), EALIGN), (dict(v=0x100004), EALIGN),
    (dict(o=HALF), EALIGN), (dict(lse=HALF), EALIGN), (dict(q_starts=HALF), EALIGN), (dict(q_tokens=2, q_token=260), EALIGN),
    (dict(o_rest=0x100008), EALIGN), (dict(k_head=68), EALIGN)]


def test_attention(lib):
    assert lib.ue5m3_attention(attention_args(), None, None) == OK and lib.ue5m3_attention(None, None, None) == EINVAL
    assert lib.ue5m3_attention(attention_args(q_starts=None, k_starts=None, sequences=3), None, None) == OK
    for kw, want in BAD_ATTENTION:
        assert lib.ue5m3_attention(attention_args(**kw), None, None) == want, kw


def test_attention_scratch(lib):
    few = dict(q_tokens=100, k_tokens=5000)
    n = lib.ue5m3_attention_scratch
    assert n(attention_args(**few)) > 0 and n(attention_args(q_tokens=100, k_tokens=100)) == 0 and n(None) == 0
    assert n(attention_args(q_tokens=-1, k_tokens=5000)) == 0 and n(attention_args(window=-1, **few)) == 0
    assert lib.ue5m3_attention(attention_args(**few), None, None) == EINVAL
    assert lib.ue5m3_attention(attention_args(**few), HALF, None) == EALIGN
    assert lib.ue5m3_attention_grad_scratch(attention_args(**few)) >= 2 * 4 * 100 * 4


def test_attention_grad(lib):
    def call(grad=None, **kw):
        a = dict(d_o=PTR, scratch=PTR, dq=PTR, dk=PTR, dv=PTR, dq_token=256, dq_head=64, dk_token=128, dk_head=64, dv_token=128, dv_head=64)
        a.update(grad or {})
        return lib.ue5m3_attention_grad(attention_args(**kw), AttentionGradC(**a), None)
    assert call() == OK and call(dict(dq=None, dk=None, dv=None)) == OK
    for kw, want in BAD_ATTENTION:
        assert call(**kw) == want, kw
    assert call(dict(dk=None)) == EINVAL and call(dict(dv=None)) == EINVAL
    for null in ("d_o", "scratch"):
        assert call({null: None}, q_tokens=1) == EINVAL
    assert call(q_tokens=1, lse=None) == EINVAL and call(q_tokens=1, o_rest=None) == EINVAL
    for odd in ("d_o", "dq", "dk", "dv"):
        assert call({odd: 0x100008}) == EALIGN
    assert call(dict(scratch=HALF)) == EALIGN and call(dict(dq_head=12)) == EALIGN and call(dict(dv_token=4)) == EALIGN
    assert lib.ue5m3_attention_grad(attention_args(), None, None) == EINVAL


def test_paged_attention(lib):
    def call(cache=None, scratch=PTR, **kw):
        a = dict(rows=0, q_heads=4, kv_heads=2, dim=64, type=BF16, scale=0.1, window=0, sinks=0, q=PTR, q_token=256, q_head=64,
                 cache=pages() if cache is None else cache, table=PTR, width=4, table_row=4, lengths=PTR, o=PTR)
        a.update(kw)
        return lib.ue5m3_paged_attention(PagedAttentionC(**a), scratch, None)
    assert call() == OK and lib.ue5m3_paged_attention(None, None, None) == EINVAL
    for kw, want in BAD_HEADS:
        assert call(**kw) == want, kw
    assert call(pages(page_size=12)) == EINVAL and call(pages(pages=-1)) == ESHAPE and call(pages(token=60)) == EALIGN
    assert call(rows=-1) == ESHAPE and call(width=-1) == ESHAPE and call(width=2 ** 27) == ESHAPE and call(rows=2, table_row=3) == ESHAPE
    assert call(pages(pages=0), rows=1) == ESHAPE and call(rows=2 ** 24, q_heads=64, kv_heads=64) == ESHAPE
    for null in ("q", "o", "lengths", "table"):
        assert call(rows=1, **{null: None}) == EINVAL, null
    assert call(pages(k=None), rows=1) == EINVAL and call(rows=1, width=1024, table_row=1024, scratch=None) == EINVAL
    assert call(rows=1, q=0x100008) == EALIGN and call(rows=1, o=HALF) == EALIGN and call(pages(v=0x100008), rows=1) == EALIGN
    assert call(rows=1, table=HALF) == EALIGN and call(rows=1, lengths=HALF) == EALIGN and call(rows=1, q_head=68) == EALIGN
    assert call(rows=1, scratch=HALF) == EALIGN
    n = lib.ue5m3_paged_attention_scratch
    assert n(0, 4, 2, 64, 1000, 0, 0) == 0 and n(1, 4, 3, 64, 1000, 0, 0) == 0 and n(1, 4, 2, 64, 64, 0, 0) == 0
    assert n(1, 32, 8, 128, 32768, 0, 0) > 0 and n(4096, 32, 8, 128, 32768, 0, 0) == 0
    assert n(1, 32, 8, 128, 2 ** 30, 2 ** 62, 2 ** 62) == n(1, 32, 8, 128, 2 ** 30, 0, 0)


def test_binding_refuses():
    """Host tensors raise before the library is called."""
    x, f = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.ones(32)
    c = torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    n = torch.zeros(4, dtype=torch.int64)
    for call in (lambda: qk_norm_rope(x, x, freqs=f), lambda: qk_norm_rope_append(x, x, x, c, c, n, freqs=f), lambda: attention(x, x, x),
                 lambda: paged_attention(x, c, c, n[None].int(), n.int()), lambda: copy_pages(c, [0], [1]),
                 lambda: PagedCache(1, 4, 12, 1, 8, device="cpu"), lambda: rotary_frequencies(7), lambda: rotary_frequencies(8, factor=0.5),
                 lambda: rotary_frequencies(8, kind="other"), lambda: rotary_frequencies(8, kind="parts"),
                 lambda: rotary_frequencies(2, factor=2.0, kind="base")):
        with pytest.raises(ValueError):
            call()


def test_no_gradients_are_dropped():
    x, c = torch.zeros(4, 2, 64, dtype=torch.bfloat16, requires_grad=True), torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    n = torch.zeros(4, dtype=torch.int64)
    for call in (lambda: qk_norm_rope_append(x, x, x, c, c, n), lambda: paged_attention(x, c, c, n[None].int(), n.int()),
                 lambda: copy_pages(x, [0], [1])):
        with pytest.raises(RuntimeError, match="no gradients"):
            call()
    half = x.detach().half().requires_grad_()
    with pytest.raises(NotImplementedError):
        attention(half, half, half)


def test_frequencies():
    """Scaled frequencies by their definitions, in 64 bits, to a rounding of fp32."""
    i = torch.arange(0, 64, 2, dtype=torch.float64)
    plain = 10000.0 ** (-i / 64)
    near = lambda a, b: ((a.double() - b).abs() <= 2.0 ** -24 * b * (1 + 2 ** -20)).all()  # noqa: E731
    make = lambda **kw: rotary_frequencies(64, device="cpu", **kw)  # noqa: E731
    assert near(make()[0], plain) and make()[1] == 1.0
    assert near(make(factor=4.0)[0], plain / 4)
    f, _ = make(factor=4.0, kind="base")
    assert f[0] == 1.0 and abs(f[-1].double() * 4 / plain[-1] - 1) < 1e-6
    f, a = make(factor=4.0, kind="parts", original=4096)
    turns = 4096 * plain / (2 * torch.pi)
    assert near(f[turns > 32], plain[turns > 32]) and near(f[turns < 1], plain[turns < 1] / 4) and abs(a - 1.1386294) < 1e-6
    between = (turns > 1) & (turns < 32)
    assert between.any() and (f[between] < plain[between]).all() and (f[between] > plain[between] / 4).all()
