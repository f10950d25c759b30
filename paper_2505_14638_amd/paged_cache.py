"""A pool of key/value pages for all layers of a model, and which sequence holds which.

The pool is one tensor [2 * layers, pages, kv_heads, page_size, head_dim] (plane 2l: keys of layer l, 2l + 1: its values).  A sequence is a list
of pages and a length; a fork shares its parent's pages, and a shared page that is not full is copied when one of its sequences
grows.  Bookkeeping is done on the host and pages are moved by w4a8_cache_copy_pages on the current stream; a call either succeeds or raises
and changes nothing.  Uploading the small index tensors that calls return keeps them out of HIP graph capture.
"""
from __future__ import annotations

import torch

from . import binding as B


class OutOfPages(RuntimeError):
    pass


class PagedCache:
    def __init__(self, layers: int, pages: int, kv_heads: int, head_dim: int, page_size: int = 16, kv_scales: torch.Tensor | None = None,
                 device: str = "cuda:0"):
        """kv_scales: None for a bf16 cache; for E4M3 bytes, float32 [layers, 2] on the device, the static scales of each layer's keys and values."""
        if min(layers, pages, kv_heads) < 1 or head_dim not in (64, 128) or page_size not in (16, 32, 64, 128, 256, 512, 1024):
            raise ValueError("layers, pages, kv_heads >= 1, head_dim 64 or 128, page_size a power of two from 16 to 1024")
        if kv_scales is not None and (kv_scales.dtype != torch.float32 or tuple(kv_scales.shape) != (layers, 2) or not kv_scales.is_contiguous()):
            raise ValueError(f"kv_scales: contiguous float32 ({layers}, 2)")
        self.page_size, self.kv_scales, self.device = page_size, kv_scales, device
        self.data = torch.empty((2 * layers, pages, kv_heads, page_size, head_dim), dtype=torch.bfloat16 if kv_scales is None else torch.uint8,
                                device=device)
        self._uses = [0] * pages                                 # sequences that hold a page
        self._free = list(range(pages - 1, -1, -1))              # the lowest is handed out first
        self._pages: dict[int, list[int]] = {}
        self._length: dict[int, int] = {}
        self._next = 0

    def layer(self, i: int):
        """(keys, values, scales or None) of a layer, as the entry points take them."""
        return self.data[2 * i], self.data[2 * i + 1], None if self.kv_scales is None else self.kv_scales[i]

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def length(self, seq: int) -> int:
        return self._length[seq]

    def open(self) -> int:
        """A new, empty sequence."""
        seq, self._next = self._next, self._next + 1
        self._pages[seq], self._length[seq] = [], 0
        return seq

    def fork(self, seq: int) -> int:
        """A new sequence of the same tokens, on the same pages."""
        pages = self._pages[seq]
        new = self.open()
        for p in pages:
            self._uses[p] += 1
        self._pages[new], self._length[new] = list(pages), self._length[seq]
        return new

    def close(self, seq: int) -> None:
        """Gives up a sequence; pages that no other one holds are free."""
        for p in self._pages[seq]:
            self._release(p)
        del self._pages[seq], self._length[seq]

    def _release(self, page: int) -> None:
        self._uses[page] -= 1
        if self._uses[page] == 0:
            self._free.append(page)

    def grow(self, seqs: list[int], counts: list[int]):
        """Room for counts[i] further tokens of seqs[i] (distinct): (positions, slots), int32 on the device, of all of them in order, as
        w4a8_rope_cache_write takes them.  positions.behind_tokens says whether any of them come behind tokens that the sequence holds already."""
        if len(set(seqs)) != len(seqs) or len(seqs) != len(counts) or any(c < 0 for c in counts):
            raise ValueError("distinct sequences with a count >= 0 each")
        own, wanted = {}, 0                                      # sequences whose last page has to become their own
        uses: dict[int, int] = {}
        for s, c in zip(seqs, counts):
            n, pages = self._length[s], self._pages[s]
            if c and n % self.page_size:
                last = pages[-1]
                if uses.setdefault(last, self._uses[last]) > 1:
                    uses[last] -= 1
                    own[s] = last
            wanted += -(-(n + c) // self.page_size) - len(pages)
        wanted += len(own)
        if wanted > len(self._free):
            raise OutOfPages(f"{wanted} pages wanted, {len(self._free)} free")
        fresh = self._free[:-wanted - 1:-1]
        copies, rest = dict(zip(own, fresh)), iter(fresh[len(own):])
        positions, slots, ends = [], [], []                      # ends: the pages of each sequence from the first that is not full on
        for s, c in zip(seqs, counts):
            n, full = self._length[s], self._length[s] // self.page_size
            end = [copies.get(s, p) for p in self._pages[s][full:]]
            while (full + len(end)) * self.page_size < n + c:
                end.append(next(rest))
            positions += range(n, n + c)
            slots += [end[j // self.page_size - full] * self.page_size + j % self.page_size for j in range(n, n + c)]
            ends.append(end)
        told = self._ints(positions), self._ints(slots)
        told[0].behind_tokens = any(c and self._length[s] for s, c in zip(seqs, counts))
        if own:
            B.cache_copy_pages(self.data, self._ints(list(own.values())), self._ints(fresh[:len(own)]))
        # the books, after all that can raise
        del self._free[len(self._free) - wanted:]
        for p in fresh:
            self._uses[p] = 1
        for old in own.values():
            self._release(old)
        for s, c, end in zip(seqs, counts, ends):
            self._pages[s][self._length[s] // self.page_size:] = end
            self._length[s] += c
        return told

    def tables(self, seqs: list[int], share: bool = True):
        """What w4a8_attention_decode takes for a batch: (tables, lengths, prefix_pages or None, prefix_length).  share: the full pages that
        all of two or more sequences begin with are the prefix, and the tables list what follows."""
        lists, lengths = [self._pages[s] for s in seqs], [self._length[s] for s in seqs]
        common = 0
        if share and len(seqs) > 1:
            most = min(n // self.page_size for n in lengths)
            while common < most and all(p[common] == lists[0][common] for p in lists):
                common += 1
        width = max([len(p) - common for p in lists] + [1])
        rows = [p[common:] + [0] * (width - len(p) + common) for p in lists]
        return (self._ints(rows).reshape(len(seqs), width), self._ints([n - common * self.page_size for n in lengths]), self._ints(lists[0][:common]) if common else None,
                common * self.page_size)

    def compact(self) -> int:
        """Moves pages so that the used ones are the lowest; returns how many those are.  Tables and slots from before are void."""
        used = sum(u > 0 for u in self._uses)
        src = [p for p in range(used, len(self._uses)) if self._uses[p] > 0]
        dst = [p for p in range(used) if self._uses[p] == 0]
        if src:
            B.cache_copy_pages(self.data, self._ints(src), self._ints(dst))
            moved = dict(zip(src, dst))
            for a, b in moved.items():
                self._uses[b], self._uses[a] = self._uses[a], 0
            for pages in self._pages.values():
                pages[:] = [moved.get(p, p) for p in pages]
        self._free = list(range(len(self._uses) - 1, used - 1, -1))
        return used

    def _ints(self, values) -> torch.Tensor:
        return torch.tensor(values, dtype=torch.int32, device=self.device)
