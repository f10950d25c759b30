"""A call of the paged cache that raises changes nothing: uploads and copies that fail, as in a stream's capture or without memory.  No GPU."""
import copy

import pytest
import torch

from paper_2505_14638_amd import binding as B
from paper_2505_14638_amd.paged_cache import PagedCache


class Refused(RuntimeError):
    pass


def books(cache):
    return copy.deepcopy((cache._uses, cache._free, cache._pages, cache._length))


@pytest.fixture
def cache(monkeypatch):
    """Two forks of a page that is not full, and a sequence of its own."""
    monkeypatch.setattr(B, "cache_copy_pages", lambda data, src, dst: data)
    cache = PagedCache(1, 12, 1, 64, 16, device="cpu")
    first, alone = cache.open(), cache.open()
    cache.grow([first, alone], [20, 40])
    cache.fork(first)
    return cache


def refuse_upload(monkeypatch, after):
    plain, calls = PagedCache._ints, []

    def ints(self, values):
        calls.append(values)
        if len(calls) > after:
            raise Refused
        return plain(self, values)
    monkeypatch.setattr(PagedCache, "_ints", ints)


@pytest.mark.parametrize("after", [0, 1, 2, 3])
def test_grow_when_an_upload_fails(cache, monkeypatch, after):
    before = books(cache)
    with monkeypatch.context() as m:
        refuse_upload(m, after)
        with pytest.raises(Refused):
            cache.grow([0, 1, 2], [3, 30, 14])
    assert books(cache) == before
    positions, slots = cache.grow([0, 1, 2], [3, 30, 14])
    assert positions.tolist() == [20, 21, 22] + list(range(40, 70)) + list(range(20, 34)) and len(set(slots.tolist())) == 47
    assert [cache.length(s) for s in range(3)] == [23, 70, 34]


def test_grow_when_a_copy_fails(cache, monkeypatch):
    def refuse(*_):
        raise Refused
    before = books(cache)
    with monkeypatch.context() as m:
        m.setattr(B, "cache_copy_pages", refuse)
        with pytest.raises(Refused):
            cache.grow([2], [1])
        assert books(cache) == before
        cache.grow([1], [1])                                     # nothing to copy


def test_grow_by_counts_that_are_none(cache):
    before = books(cache)
    for counts in ([1, 1.5], [1, "2"], [1, None]):
        with pytest.raises((TypeError, ValueError)):
            cache.grow([0, 1], counts)
        assert books(cache) == before


def test_compact_when_an_upload_or_a_copy_fails(cache, monkeypatch):
    cache.close(0)
    cache.grow([2], [100])
    cache.close(1)
    for after in (0, 1):
        before = books(cache)
        with monkeypatch.context() as m:
            refuse_upload(m, after)
            with pytest.raises(Refused):
                cache.compact()
        assert books(cache) == before
    assert cache.compact() == 8 and cache.length(2) == 120


def test_pages_and_slots_are_the_same_numbers(cache):
    """Which pages a call hands out, in which order: copies first, then those that follow, the lowest free one first."""
    positions, slots = cache.grow([0, 2, 1], [13, 1, 8])
    assert cache._pages == {0: [0, 5, 6], 2: [0, 1], 1: [2, 3, 4]}
    assert slots.tolist() == [5 * 16 + i for i in range(4, 16)] + [6 * 16] + [1 * 16 + 4] + [4 * 16 + i for i in range(8, 16)]
    assert torch.equal(positions, torch.tensor(list(range(20, 33)) + [20] + list(range(40, 48)), dtype=torch.int32))
