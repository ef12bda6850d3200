"""Attention over a paged cache and copies of its pages, on the GPU: against 64 bits,
lengths from none on, pages that end inside a tile, windows and sinks, parts, bad
page numbers; the cache's tables, forks and compaction; a prompt and its decoding
together."""

import pytest
import torch

import attention_model as model
from gpu_util import say
from paper_2609_02846_amd.attention import attention, paged_attention
from paper_2609_02846_amd.paged import PagedCache, copy_pages
from paper_2609_02846_amd.rotary import qk_norm_rope, qk_norm_rope_append, rotary_frequencies

pytestmark = pytest.mark.gpu


def rand(seed, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def filled(lens, Hk, D, page, dtype, seed=0, hnd=True, width=None):
    """(k_cache, v_cache, table, lengths): what no sequence has is NaN."""
    need = [-(-n // page) for n in lens]
    P = sum(need) + 2
    store = torch.full((2, P, Hk, page, D) if hnd else (2, P, page, Hk, D), float("nan"), dtype=dtype, device="cuda")
    kc, vc = (store[i].transpose(1, 2) if hnd else store[i] for i in (0, 1))
    order = torch.randperm(P, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((len(lens), width or max(max(need), 1)), -1, dtype=torch.int32)
    for b, n in enumerate(lens):
        for i in range(need[b]):
            p = order.pop()
            table[b, i] = p
            m = min(page, n - i * page)
            kc[p, :m], vc[p, :m] = rand(seed + 7 * p + 1, m, Hk, D, dtype=dtype), rand(seed + 7 * p + 2, m, Hk, D, dtype=dtype)
    return kc, vc, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()


def check(lens, Hq, Hk, D, page, dtype=torch.bfloat16, window=0, sinks=0, hnd=True, width=None, seed=0):
    say("paged", lens, Hq, Hk, D, page, dtype, window, sinks, hnd)
    kc, vc, table, lengths = filled(lens, Hk, D, page, dtype, seed, hnd, width)
    q = 1.5 * rand(seed + 1000003, len(lens), Hq, D, dtype=dtype)
    o = paged_attention(q, kc, vc, table, lengths, window=window, sinks=sinks)
    for b, n in enumerate(lens):
        at = torch.arange(n).cuda()
        rows = table[b].long()[at // page], at % page
        want = model.Sequence(q[b:b + 1], kc[rows], vc[rows], D ** -0.5, window=window, sinks=sinks)
        model.within(o[b:b + 1], want.o.transpose(0, 1), want.o_bound().transpose(0, 1), (b, n))
    assert torch.equal(o, paged_attention(q, kc, vc, table, lengths, window=window, sinks=sinks))


@pytest.mark.parametrize("page", [1, 8, 16, 32, 64, 256])
def test_lengths(page):
    check([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 0, 300], 4, 2, 64, page)
    check([0, 7, 100, 513], 2, 1, 128, page, torch.float16, hnd=False)


@pytest.mark.parametrize("heads", [(1, 1), (32, 8), (8, 1), (16, 1), (17, 1), (40, 1), (9, 3)])
@pytest.mark.parametrize("D", [8, 64, 80, 128])
def test_heads(heads, D):
    check([100, 37, 1], *heads, D, 16)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (32, 40), (64, 0), (100, 4), (300, 70), (10 ** 9, 5), (2 ** 40, 2 ** 40)])
def test_windows_and_sinks(window, sinks):
    check([0, 1, 5, 33, 64, 101, 150, 700, 1500], 4, 2, 64, 16, window=window, sinks=sinks)


def test_parts():
    """Long rows in several parts, beside short ones that leave parts empty."""
    check([5000, 0, 3, 260, 4097], 8, 2, 128, 16)
    check([20011], 4, 1, 64, 64)
    check([3000], 2, 1, 128, 16, window=900, sinks=5)
    check([10, 20], 4, 2, 64, 16, width=500)         # a wide table, short rows


def test_bad_pages():
    """A number outside the cache, or a length past the table, makes its row NaN, others
    as they were; one that is not needed does nothing."""
    lens = [100, 64, 300]
    kc, vc, table, lengths = filled(lens, 2, 64, 16, torch.bfloat16)
    q = rand(5, 3, 4, 64)
    good = paged_attention(q, kc, vc, table, lengths)
    for bad in (-1, kc.shape[0], 2 ** 31 - 1, -(2 ** 31)):
        t = table.clone()
        t[1, 3] = bad
        o = paged_attention(q, kc, vc, t, lengths)
        assert torch.isnan(o[1]).all() and torch.equal(o[0], good[0]) and torch.equal(o[2], good[2])
        t = table.clone()
        t[0, 0] = bad                                # out of the window
        assert torch.isfinite(paged_attention(q, kc, vc, t, lengths, window=50)).all()
    for n in (16 * table.shape[1] + 1, 2 ** 31 - 1):
        long = lengths.clone()
        long[1] = n
        assert torch.isnan(paged_attention(q, kc, vc, table.clamp_min(0), long)[1]).all()
    long[1] = -3
    assert not paged_attention(q, kc, vc, table, long)[1].any()


def test_offsets_past_32_bits():
    """Pages beyond 2^32 bytes of a cache."""
    P, page, Hk, D = 2200, 1024, 8, 128
    say("large cache", P * page * Hk * D * 2)
    k = torch.zeros(P, Hk, page, D, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    v = torch.zeros_like(k)
    last = P - 1
    k[last], v[last], k[0], v[0] = (rand(i, page, Hk, D) for i in range(4))
    q = rand(9, 2, 32, D)
    table = torch.tensor([[last, 0], [0, last]], dtype=torch.int32).cuda()
    lengths = torch.tensor([1500, 2048], dtype=torch.int32).cuda()
    o = paged_attention(q, k, v, table, lengths)
    for b, n in enumerate(lengths.tolist()):
        kk = torch.cat([k[t] for t in table[b].tolist()])[:n]
        vv = torch.cat([v[t] for t in table[b].tolist()])[:n]
        want = model.Sequence(q[b:b + 1], kk, vv, D ** -0.5)
        model.within(o[b:b + 1], want.o.transpose(0, 1), want.o_bound().transpose(0, 1), b)
    copy_pages(v.transpose(1, 2), [0], [last])
    assert torch.equal(v[last], v[0]) and v[0].any()


@pytest.mark.parametrize("shape,dim,dtype", [((4, 2, 20, 3, 8, 16), 2, torch.bfloat16), ((50, 7), 0, torch.float32),
                                             ((3, 600, 5), 1, torch.float16), ((2, 9, 4096, 3), 1, torch.int32), ((9, 16), 0, torch.float8_e4m3fn)])
def test_copies(shape, dim, dtype):
    n = shape[dim]
    x = torch.randint(-100, 100, shape, generator=torch.Generator().manual_seed(1)).float().to(dtype).cuda()
    order = torch.randperm(n, generator=torch.Generator().manual_seed(2)).tolist()
    half = n // 2
    src, dst = [order[i // 2] for i in range(half)], order[half:2 * half]       # pages copied twice
    want = x.clone()
    bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()]
    w, s = want.view(bits), x.view(bits)
    for a, b in zip(src, dst):
        w.select(dim, b).copy_(s.select(dim, a))
    copy_pages(x, src, torch.tensor(dst), dim=dim)
    assert torch.equal(x.view(bits), w)
    copy_pages(x, [], [], dim=dim)
    assert torch.equal(x.view(bits), w)


def test_cache_forks_and_compaction():
    """Tables of sequences that grow, fork, end and move, against a list of each one's
    tokens."""
    c = PagedCache(2, 40, 4, 1, 8)
    tokens, counter = {}, [0]

    def grow(*pairs):
        seqs, counts = [p[0] for p in pairs], [p[1] for p in pairs]
        slots = c.extend(seqs, counts)
        values = torch.arange(counter[0], counter[0] + len(slots), device="cuda").to(torch.bfloat16)
        counter[0] += len(slots)
        rows = values.view(-1, 1, 1).expand(-1, 1, 8).contiguous()
        for layer in range(2):
            qk_norm_rope_append(None, rows + 64 * layer, -rows, *c.layer(layer), slots, eps=None)
        at = 0
        for s, n in zip(seqs, counts):
            tokens[s] = tokens.get(s, []) + values[at:at + n].tolist()
            at += n

    def verify():
        torch.cuda.synchronize()
        assert c.free_pages() == 40 - len({p for s in tokens for p in c._sequences[s][0]})
        if not tokens:
            return
        table, lengths = c.tables(list(tokens))
        assert lengths.tolist() == [len(t) for t in tokens.values()]
        for layer in range(2):
            k, v = c.layer(layer)
            for row, t in zip(table.tolist(), tokens.values()):
                got = [k[row[i // 4], i % 4, 0, 3].item() for i in range(len(t))]
                assert got == [(torch.tensor(x, dtype=torch.bfloat16) + 64 * layer).item() for x in t]
                assert [v[row[i // 4], i % 4, 0, 0].item() for i in range(len(t))] == [-x for x in t]
    a, b = c.open(), c.open()
    grow((a, 6), (b, 3))
    verify()
    d = c.fork(a)
    tokens[d] = list(tokens[a])
    e = c.fork(a)
    tokens[e] = list(tokens[a])
    verify()
    grow((d, 1), (a, 2), (e, 5))                     # each takes a page of its own, the last keeps the old one
    verify()
    grow((b, 1), (d, 9))
    c.close(a)
    del tokens[a]
    verify()
    used = c.compact()
    assert used == 40 - c.free_pages() and max(p for s in tokens for p in c._sequences[s][0]) == used - 1
    verify()
    f = c.fork(b)
    tokens[f] = list(tokens[b])
    with pytest.raises(MemoryError):
        c.extend([f, d], [1, 1000])
    verify()
    grow((f, 2), (b, 0))
    for s in list(tokens):
        c.close(s)
        del tokens[s]
    verify()
    assert c.compact() == 0


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
def test_prompt_and_decoding_together(window, sinks):
    """A prompt's rotation, attention and cache, a fork, and tokens decoded one by one
    in both, against the attention of whole sequences: the same rows but for the order
    of sums (bounded as each is, twice)."""
    Hq, Hk, D, prompt, steps = 8, 2, 64, 75, 6
    x = rand(1, 2, prompt + steps, Hq + 2 * Hk, D)
    x[1, :prompt] = x[0, :prompt]                    # one prompt, two continuations
    w = (1 + 0.1 * rand(2, D).float()).to(torch.bfloat16)
    f = rotary_frequencies(D)[0]
    whole = [t.contiguous() for t in x.split([Hq, Hk, Hk], dim=2)]
    q, k = qk_norm_rope(whole[0], whole[1], w, w, None, f)
    want = attention(q, k, whole[2], window=window, sinks=sinks)
    c = PagedCache(1, 30, 8, Hk, D)
    kc, vc = c.layer(0)
    a = c.open()
    first = x[0, :prompt]
    pq, pk = qk_norm_rope(first[:, :Hq], first[:, Hq:Hq + Hk], w, w, None, f)
    qk_norm_rope_append(None, pk, first[:, Hq + Hk:], kc, vc, c.extend([a], [prompt]), eps=None)
    assert torch.equal(attention(pq, pk, first[:, Hq + Hk:], window=window, sinks=sinks), want[0, :prompt])
    b = c.fork(a)
    for t in range(prompt, prompt + steps):
        token = x[:, t]
        slots = c.extend([a, b], [1, 1])
        qt = qk_norm_rope_append(token[:, :Hq], token[:, Hq:Hq + Hk], token[:, Hq + Hk:], kc, vc, slots, w, w,
                                 torch.full((2,), t).cuda(), f)
        assert torch.equal(qt, q[:, t])
        table, lengths = c.tables([a, b])
        o = paged_attention(qt, kc, vc, table, lengths, window=window, sinks=sinks)
        for i in range(2):
            ref = model.Sequence(q[i, t:t + 1], k[i, :t + 1], whole[2][i, :t + 1], D ** -0.5, window=window, sinks=sinks)
            model.within(o[i:i + 1], ref.o.transpose(0, 1), ref.o_bound().transpose(0, 1), (t, i))
            model.within(o[i:i + 1], want[i, t:t + 1].double(), 2 * ref.o_bound().transpose(0, 1), (t, i, "whole"))


def test_replays_of_captured_decoding():
    """Two graphs captured after one another, replayed in turn on changed tables and
    lengths."""
    kc, vc, table, lengths = filled([5000, 300], 2, 64, 16, torch.bfloat16)
    q = rand(3, 2, 8, 64)
    held = [q.clone(), lengths.clone()]
    graphs, outs = [], []
    for window in (0, 700):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(paged_attention(held[0], kc, vc, table, held[1], window=window, sinks=2))
        graphs.append(g)
    for i in range(4):
        held[0].copy_(q * (i + 1) / 2)
        held[1].copy_(torch.tensor([5000 - 1111 * i, 300 - 99 * i], dtype=torch.int32))
        want = [paged_attention(held[0], kc, vc, table, held[1], window=w, sinks=2) for w in (0, 700)]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), i
