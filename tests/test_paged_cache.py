"""The bookkeeping of the paged cache against sequences kept as plain lists, with the page copies done by indexing.  No GPU."""
import random

import pytest
import torch

from paper_2505_14638_amd import binding as B
from paper_2505_14638_amd.paged_cache import OutOfPages, PagedCache


@pytest.fixture(autouse=True)
def copies_by_indexing(monkeypatch):
    def copy(cache, src, dst):
        src, dst = src.tolist(), dst.tolist()
        assert len(set(dst)) == len(dst) == len(src) and not set(src) & set(dst)
        cache[:, dst] = cache[:, src].clone()
        return cache
    monkeypatch.setattr(B, "cache_copy_pages", copy)


def read(cache, tables, lengths, prefix_pages, prefix_length):
    """The tokens that a decode call would see, by the first channel of plane 0 (whole numbers here)."""
    flat = cache.data[0, :, 0, :, 0]
    got = []
    for row, n in zip(tables.tolist(), lengths.tolist()):
        pages = ([] if prefix_pages is None else prefix_pages.tolist())
        front = flat[pages].reshape(-1)[:prefix_length]
        got.append(torch.cat([front, flat[row].reshape(-1)[:n]]).int().tolist())
    return got


@pytest.mark.parametrize("seed", range(8))
def test_against_plain_lists(seed):
    rng = random.Random(seed)
    page = rng.choice((16, 32))
    cache = PagedCache(2, 24, 1, 64, page, kv_scales=torch.ones(2, 2) if seed % 2 else None, device="cpu")
    plain, counter, refused = {}, 0, 0
    for _ in range(300):
        what = rng.random()
        if what < 0.15 or not plain:
            plain[cache.open()] = []
        elif what < 0.3:
            seq = rng.choice(list(plain))
            plain[cache.fork(seq)] = list(plain[seq])
        elif what < 0.42:
            seq = rng.choice(list(plain))
            cache.close(seq)
            del plain[seq]
        elif what < 0.5:
            used = cache.compact()
            assert used + cache.free_pages == 24
            assert sorted(cache._free) == list(range(used, 24))
        else:
            seqs = rng.sample(list(plain), rng.randint(1, len(plain)))
            counts = [rng.choice((0, 1, 1, 1, page, rng.randint(0, 40))) for _ in seqs]
            before = ({s: list(p) for s, p in cache._pages.items()}, dict(cache._length), list(cache._uses), list(cache._free))
            try:
                positions, slots = cache.grow(seqs, counts)
            except OutOfPages:
                refused += 1
                assert before == (cache._pages, cache._length, cache._uses, cache._free)
                continue
            assert len(set(slots.tolist())) == len(slots)
            values = [(counter + i) % 200 for i in range(sum(counts))]
            counter += len(values)
            for s, v in zip(slots.tolist(), values):
                cache.data[:, s // page, :, s % page] = v
            at = 0
            for seq, c in zip(seqs, counts):
                assert positions[at:at + c].tolist() == list(range(len(plain[seq]), len(plain[seq]) + c))
                plain[seq] += values[at:at + c]
                at += c
        seqs = list(plain)
        for share in (True, False):
            if seqs:
                assert read(cache, *cache.tables(seqs, share)) == [plain[s] for s in seqs]
        assert all(cache.length(s) == len(plain[s]) for s in seqs)
        held = [p for s in seqs for p in cache._pages[s]]
        assert all(cache._uses[p] == held.count(p) for p in range(24)) and sorted(set(held) | set(cache._free)) == list(range(24))
    assert refused > 0


def test_forks_share_their_prefix():
    cache = PagedCache(1, 40, 1, 64, 16, device="cpu")
    first = cache.open()
    cache.grow([first], [100])
    others = [cache.fork(first) for _ in range(3)]
    used = 40 - cache.free_pages
    assert used == 7
    cache.grow(others, [1, 1, 20])
    assert 40 - cache.free_pages == used + 3 + 1                 # each copies the page that is not full
    tables, lengths, prefix_pages, prefix_length = cache.tables([first] + others)
    assert prefix_length == 96 and len(prefix_pages) == 6 and lengths.tolist() == [4, 5, 5, 24] and tables.shape == (4, 2)
    assert cache.tables([first])[3] == 0 and cache.tables([first] + others, share=False)[3] == 0


def test_refusals():
    for bad in (dict(layers=0), dict(pages=0), dict(kv_heads=0), dict(head_dim=96), dict(page_size=24), dict(kv_scales=torch.ones(3, 2)),
                dict(kv_scales=torch.ones(2, 2, dtype=torch.float64))):
        with pytest.raises(ValueError):
            PagedCache(**{**dict(layers=2, pages=4, kv_heads=1, head_dim=64, device="cpu"), **bad})
    cache = PagedCache(1, 4, 1, 64, device="cpu")
    seq = cache.open()
    for seqs, counts in (([seq, seq], [1, 1]), ([seq], [1, 2]), ([seq], [-1])):
        with pytest.raises(ValueError):
            cache.grow(seqs, counts)
    with pytest.raises(OutOfPages):
        cache.grow([seq], [65])
    with pytest.raises(KeyError):
        cache.grow([seq + 1], [1])
    assert cache.length(seq) == 0 and cache.free_pages == 4


def test_an_empty_batch():
    cache = PagedCache(1, 4, 1, 64, device="cpu")
    positions, slots = cache.grow([], [])
    tables, lengths, prefix_pages, prefix_length = cache.tables([])
    assert positions.numel() == slots.numel() == lengths.numel() == prefix_length == 0 and prefix_pages is None and tuple(tables.shape) == (0, 1)
    assert cache.compact() == 0 and cache.free_pages == 4
