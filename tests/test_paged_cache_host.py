"""PagedCache when the copy of a shared page fails: nothing has changed (on the host, with
a stand-in for the copy)."""

import copy

import pytest
import torch

import paper_2609_02846_amd.paged as paged
from paper_2609_02846_amd.paged import PagedCache


def state(c):
    return copy.deepcopy((c._sequences, c._uses, c._free, c._next))


def forked():
    c = PagedCache(1, 12, 4, 1, 8, device="cpu")
    a, other = c.open(), c.open()
    c.extend([a, other], [6, 4])                     # (no page is shared: nothing is copied)
    return c, a, other, c.fork(a)


def test_a_failed_copy_changes_nothing(monkeypatch):
    c, a, other, b = forked()
    before = state(c)
    calls = []

    def fail(*args, **kw):
        calls.append(args)
        raise RuntimeError("no copy")
    with monkeypatch.context() as m:
        m.setattr(paged, "copy_pages", fail)
        with pytest.raises(RuntimeError, match="no copy"):
            c.extend([other, b, a], [9, 1, 3])
    assert calls and state(c) == before
    with pytest.raises(ValueError):                  # the copy itself, of a cache on the host
        c.extend([b], [1])
    assert state(c) == before
    with monkeypatch.context() as m:
        m.setattr(paged, "copy_pages", fail)
        c.close(other)
        before = state(c)
        with pytest.raises(RuntimeError, match="no copy"):
            c.compact()
    assert state(c) == before


def test_a_failed_transfer_of_the_slots_changes_nothing(monkeypatch):
    c, a, other, b = forked()
    before = state(c)

    def fail(*args, **kw):
        raise RuntimeError("no memory")
    with monkeypatch.context() as m:
        m.setattr(paged, "copy_pages", lambda *args, **kw: None)
        m.setattr(torch, "tensor", fail)
        with pytest.raises(RuntimeError, match="no memory"):
            c.extend([a, b], [3, 3])
    assert state(c) == before


def test_extend_after_a_fork(monkeypatch):
    """Which pages are copied, in which order sequences get theirs, and the slots."""
    c, a, other, b = forked()
    d = c.fork(a)
    calls = []
    monkeypatch.setattr(paged, "copy_pages", lambda cache, src, dst, dim: calls.append((list(src), list(dst), dim)))
    old, last = list(c._sequences[a][0]), c._sequences[a][0][1]
    slots = c.extend([b, a, other, d], [3, 0, 5, 1]).tolist()
    pages = {s: c._sequences[s][0] for s in (a, b, d, other)}
    assert pages[a] == old and [c.length(s) for s in (a, b, d, other)] == [6, 9, 7, 9]
    assert calls == [([last, last], [pages[b][1], pages[d][1]], 2)]
    assert slots == [pages[b][1] * 4 + 2, pages[b][1] * 4 + 3, pages[b][2] * 4, *(pages[other][1] * 4 + i for i in range(4)),
                     pages[other][2] * 4, pages[d][1] * 4 + 2]
    used = [p for s in pages.values() for p in s]
    assert [c._uses[p] for p in range(12)] == [used.count(p) for p in range(12)]
    assert sorted(c._free) == [p for p in range(12) if not c._uses[p]]
