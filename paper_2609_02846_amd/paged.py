"""The pages of a cache of keys and values: which sequence has which, sharing
after a fork, copies on writing, compaction."""

import array
import ctypes

import torch
from torch.autograd.graph import increment_version

from . import _check, _numel, _stream, load_library
from .operators import recorded
from .rotary import _on_device


def _page_numbers(pages, name):
    if isinstance(pages, torch.Tensor):
        if pages.is_cuda:
            raise ValueError(f"{name} must be on the host")
        pages = pages.tolist()
    try:
        return array.array("i", pages)
    except (TypeError, OverflowError) as e:
        raise ValueError(f"{name} must be page numbers") from e


def copy_pages(cache, src, dst, dim=0):
    """Copies page ``src``[i] of ``cache`` to ``dst``[i], in place, pages being its slices
    along ``dim``, all that lies before ``dim`` (layers, keys and values) at once.
    ``cache``: contiguous, of any type; ``src``, ``dst``: lists or host tensors.  No page may
    be in ``dst`` twice, or in both (see ue5m3_copy_pages)."""
    if recorded(cache):
        raise RuntimeError("copy_pages has no gradients: call it under torch.no_grad()")
    _on_device(cache, "cache")
    if not cache.is_contiguous() or not 0 <= dim < cache.dim():
        raise ValueError("cache must be contiguous, with pages along one of its dimensions")
    src, dst = _page_numbers(src, "src"), _page_numbers(dst, "dst")
    if len(src) != len(dst):
        raise ValueError(f"{len(src)} pages to copy to {len(dst)}")
    pages = cache.shape[dim]
    page = _numel(cache.shape[dim + 1:]) * cache.element_size()
    numbers = [(ctypes.c_int32 * len(a)).from_buffer(a) if len(a) else None for a in (src, dst)]
    _check(load_library().ue5m3_copy_pages(cache.data_ptr(), _numel(cache.shape[:dim]), pages * page, pages, page, *numbers,
                                           len(src), _stream()), "ue5m3_copy_pages")
    increment_version(cache)                         # (autograd finds out where it has saved it)


class PagedCache:
    """Keys and values of several sequences, in all layers, in pages of ``page_size``
    tokens (a power of two): ``storage`` [layers, 2, pages, kv_heads, page_size, dim], a
    head's rows of a page together.

    The tables are on the host.  ``extend`` makes room for new tokens and says where
    they go, ``layer`` and ``tables`` are what ``qk_norm_rope_append`` and
    ``paged_attention`` take.  A fork shares its pages with the sequence that it
    comes from; a page that is not full is copied when one of them grows.  Copies
    run on the current stream: use the cache on one."""

    def __init__(self, layers, pages, page_size, kv_heads, dim, dtype=torch.bfloat16, device="cuda"):
        if page_size < 1 or page_size & (page_size - 1):
            raise ValueError("pages hold a power of two of tokens")
        self.page_size, self.pages = int(page_size), int(pages)
        self.storage = torch.zeros((layers, 2, pages, kv_heads, page_size, dim), dtype=dtype, device=device)
        self._free = list(range(self.pages))[::-1]
        self._uses = [0] * self.pages
        self._sequences, self._next = {}, 0          # number -> [pages, length]

    def layer(self, i):
        """(k_cache, v_cache) of layer i, [pages, page_size, kv_heads, dim]."""
        return self.storage[i, 0].transpose(1, 2), self.storage[i, 1].transpose(1, 2)

    def open(self):
        """A new sequence of no tokens; returns its number."""
        self._sequences[self._next] = [[], 0]
        self._next += 1
        return self._next - 1

    def length(self, sequence):
        return self._sequences[sequence][1]

    def free_pages(self):
        return len(self._free)

    def fork(self, sequence):
        """A sequence with the same tokens, on the same pages; returns its number."""
        pages, length = self._sequences[sequence]
        for p in pages:
            self._uses[p] += 1
        new = self.open()
        self._sequences[new] = [list(pages), length]
        return new

    def close(self, sequence):
        """Ends a sequence; pages that no other has are free again."""
        for p in self._sequences.pop(sequence)[0][::-1]:
            self._uses[p] -= 1
            if self._uses[p] == 0:
                self._free.append(p)

    def extend(self, sequences, counts):
        """Makes room for counts[i] new tokens of each of ``sequences`` (different
        ones); returns their slots, one sequence after the other (int64, on the
        device).  Raises MemoryError where pages lack.  Where it raises, nothing has
        changed."""
        sequences, counts = list(sequences), [int(c) for c in counts]
        if len(set(sequences)) != len(sequences) or len(counts) != len(sequences) or min(counts, default=0) < 0:
            raise ValueError("each sequence once, with a count that is not negative")
        size, plan, need = self.page_size, [], 0
        uses = {}                                    # of pages that this call gives up
        for s, c in zip(sequences, counts):
            pages, length = self._sequences[s]
            shared = None
            if c and length % size:                  # tokens go to a page that others have, too
                last = pages[length // size]
                left = uses.get(last, self._uses[last])
                if left > 1:
                    shared, uses[last] = last, left - 1
            new = -(-(length + c) // size) - len(pages)
            plan.append((s, c, shared, new))
            need += new + (shared is not None)
        if need > len(self._free):
            raise MemoryError(f"{need} pages needed, {len(self._free)} free")
        # what can fail comes first, with pages that are free as yet (the last one is taken first)
        kept = len(self._free) - need
        free = reversed(self._free[kept:])
        src, dst, slots, tails = [], [], [], []
        for s, c, shared, new in plan:
            pages, length = self._sequences[s]
            at = length // size                      # what changes: the pages from here on
            tail = pages[at:]
            if shared is not None:
                tail[0] = next(free)
                src.append(shared)
                dst.append(tail[0])
            if new > 0:
                tail += [next(free) for _ in range(new)]
            tails.append((at, tail))
            slots += [tail[t // size - at] * size + t % size for t in range(length, length + c)]
        if src:
            copy_pages(self.storage, src, dst, dim=2)
        slots = torch.tensor(slots, dtype=torch.int64, device=self.storage.device)
        for p in self._free[kept:]:
            self._uses[p] = 1
        del self._free[kept:]
        for p in src:
            self._uses[p] -= 1
        for (s, c, _, _), (at, tail) in zip(plan, tails):
            entry = self._sequences[s]
            entry[0][at:] = tail
            entry[1] += c
        return slots

    def tables(self, sequences):
        """(table, lengths) of ``sequences`` for ``paged_attention`` (int32, on the
        device); past a sequence's pages the table holds -1."""
        rows = [self._sequences[s] for s in sequences]
        width = max([len(p) for p, _ in rows], default=0)
        table = [p + [-1] * (width - len(p)) for p, _ in rows]
        device = self.storage.device
        return (torch.tensor(table, dtype=torch.int32, device=device).view(len(rows), width),
                torch.tensor([n for _, n in rows], dtype=torch.int32, device=device))

    def compact(self):
        """Moves the pages in use to the lowest numbers; returns how many there are.
        Tables made before no longer hold."""
        used = self.pages - len(self._free)
        holes = [p for p in range(used) if self._uses[p] == 0]
        high = [p for p in range(used, self.pages) if self._uses[p]]
        copy_pages(self.storage, high, holes, dim=2)
        to = dict(zip(high, holes))
        for a, b in to.items():
            self._uses[a], self._uses[b] = 0, self._uses[a]
        for entry in self._sequences.values():
            entry[0] = [to.get(p, p) for p in entry[0]]
        self._free = list(range(used, self.pages))[::-1]
        return used
