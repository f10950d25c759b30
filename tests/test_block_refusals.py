"""What a decoder block refuses before anything reaches the GPU.  No GPU."""
import pytest
import torch

from paper_2505_14638_amd import binding as B
from paper_2505_14638_amd.block import DecoderBlock, rotary_table
from paper_2505_14638_amd.paged_cache import PagedCache


def test_a_prompt_behind_cached_tokens_is_refused(monkeypatch):
    """Its rows would take the right positions and attend to each other alone."""
    monkeypatch.setattr(B, "cache_copy_pages", lambda data, src, dst: data)
    blk = DecoderBlock(512, 768, 8, 2, rotary_table(64, 64, device="cpu"), device="cpu")
    cache = PagedCache(1, 8, 2, 64, device="cpu")
    first, second = cache.open(), cache.open()
    assert not cache.grow([first], [20])[0].behind_tokens
    fork = cache.fork(first)
    for seqs, counts, behind in (([first], [3], True), ([second, fork], [4, 4], True), ([first, cache.open()], [0, 4], False), ([second], [0], False)):
        positions, slots = cache.grow(seqs, counts)
        assert positions.behind_tokens == behind
        if behind:
            with pytest.raises(ValueError, match="holds tokens"):
                blk.forward_prompt(torch.zeros((sum(counts), 512), dtype=torch.bfloat16), torch.tensor([0, sum(counts)], dtype=torch.int32), positions, slots,
                                   cache.layer(0))
