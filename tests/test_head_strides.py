"""Strides of a dimension of one element, which reach nothing: no call is refused for
them, and no copy keeps them (on the host; nothing is enqueued)."""

import os

import pytest
import torch

import paper_2609_02846_amd as ue
from paper_2609_02846_amd import AttentionC, PagedAttentionC, PagesC, build, rotary

OK, EALIGN = ue.UE5M3_OK, ue.UE5M3_EALIGN
PTR = 0x100000                                       # aligned, never dereferenced
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ue.LIB_PATH):
        build.build(verbose=False)
    return ue.load_library()


@pytest.fixture
def host(monkeypatch):
    monkeypatch.setattr(rotary, "_on_device", lambda t, name: t)


def views():
    """[tokens, heads, dim] of one token or one head, at odd pitches and from transposes."""
    return {"one head": torch.randn(5, 64, 1).to(BF16).transpose(1, 2),
            "one token, one head": torch.randn(4, 1, 132).to(BF16)[:1, :, :64],
            "one token of several": torch.randn(4, 100).to(BF16)[2:3, :96].view(1, 1, 96),
            "one token, heads apart": torch.randn(3, 2, 68).to(BF16)[:1, :, :64],
            "a batch of one token": torch.randn(2, 1, 1, 200).to(BF16)[:1, ..., :128],
            "batches of one token": torch.randn(3, 1, 4, 72).to(BF16)[..., :64],
            "not aligned": torch.randn(5 * 64 + 1).to(BF16)[1:].view(5, 1, 64)}


@pytest.mark.parametrize("name", list(views()))
@pytest.mark.parametrize("dense", [True, False])
def test_layouts(host, name, dense):
    t = views()[name]
    r, tokens, token, head = rotary.head_rows(t, "q", (BF16,), dense)
    assert tokens == t.shape[:-2].numel()
    assert not dense or (token % 8 == 0 and head % 8 == 0 and r.data_ptr() % 16 == 0)
    got = r.as_strided((tokens, t.shape[-2], t.shape[-1]), (token, head, 1))
    assert torch.equal(got, t.reshape(got.shape))


def test_no_copy_is_made_for_a_stride_that_reaches_nothing(host):
    for name in ("one head", "one token, one head"):
        t = views()[name]
        assert t.data_ptr() % 16 or rotary.head_rows(t, "q", (BF16,), True)[0] is t


def test_caches(host):
    """One page at an odd pitch, pages of one token, one head."""
    for shape, stride in (((1, 16, 2, 64), (2052, 128, 64, 1)), ((3, 1, 2, 64), (128, 7, 64, 1)), ((3, 16, 1, 64), (1024, 64, 1, 1))):
        k, v = (torch.zeros(10000, dtype=BF16).as_strided(shape, s) for s in (stride, torch.empty(shape).stride()))
        p, q = rotary.cache_arguments(k, k, 8), rotary.cache_arguments(k, v, 8)
        strides = [s if n > 1 else 0 for n, s in zip(shape, stride)][:3]
        assert [p.page, p.token, p.head] == strides == [q.page, q.token, q.head]
    k = torch.zeros(10000, dtype=BF16).as_strided((2, 16, 2, 64), (2052, 128, 64, 1))
    with pytest.raises(ValueError, match="multiples of 8"):
        rotary.cache_arguments(k, k, 8)
    with pytest.raises(ValueError, match="strides"):
        rotary.cache_arguments(k, torch.zeros(2, 16, 2, 64, dtype=BF16))


def test_library(lib):
    """Calls of no queries, which end before anything is enqueued."""
    def attention(**kw):
        a = dict(q_tokens=0, k_tokens=0, sequences=1, q_starts=PTR, k_starts=PTR, q_heads=1, kv_heads=1, dim=64, type=0, causal=1, scale=0.1,
                 q=PTR, k=PTR, v=PTR, q_token=64, q_head=64, k_token=64, k_head=64, v_token=64, v_head=64, o=PTR)
        a.update(kw)
        return lib.ue5m3_attention(AttentionC(**a), None, None)
    assert attention(q_token=100, q_head=1, k_head=3, v_head=5) == OK
    assert attention(k_tokens=1, k_token=100, v_token=33) == OK
    assert attention(k_tokens=2, k_token=100) == EALIGN and attention(k_tokens=2, v_token=100) == EALIGN
    assert attention(q_heads=2, q_head=100) == EALIGN and attention(q_heads=2, kv_heads=2, v_head=100) == EALIGN

    def paged(kv_heads=1, **kw):
        c = dict(k=PTR, v=PTR, pages=10, page_size=16, page=1024, token=64, head=64)
        c.update(kw)
        a = PagedAttentionC(rows=0, q_heads=2, kv_heads=kv_heads, dim=64, type=0, scale=0.1, q=PTR, q_token=3, q_head=64, cache=PagesC(**c))
        return lib.ue5m3_paged_attention(a, None, None)
    assert paged(pages=1, page=100) == OK and paged(page_size=1, token=7) == OK and paged(head=1) == OK
    assert paged(page=100) == EALIGN and paged(token=100) == EALIGN and paged(kv_heads=2, head=100) == EALIGN
