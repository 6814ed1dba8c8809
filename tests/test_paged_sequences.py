"""Sequences and lengths that a cache does not have, on the host."""
import pytest
import torch

from paper_2601_03700_amd.model import PagedKVCache


def cache(n_seq=3, n_pages=9, page=4, max_pages=3, kv="bf16"):
    return PagedKVCache(2, 2, 16, n_seq, n_pages, page, max_pages, kv, "cpu")


def test_slots_of_sequences_outside_the_table():
    """The slot for no one, as for a token without a page; not another sequence's, no error that
    would be one of the device."""
    c = cache()
    c.reserve(12)
    pos = torch.tensor([0, 0, 5, 11, 3], dtype=torch.int32)
    seq = torch.tensor([-1, 3, 2 ** 31 - 1, -2 ** 31, 2], dtype=torch.int32)
    spare = c.n_slots - 1
    assert c.slots(pos, seq).tolist() == [spare] * 4 + [int(c.page_table[2, 0]) * 4 + 3]


@pytest.mark.parametrize("seq", [-1, -3, 3, 100])
def test_sequences_outside_the_cache_have_no_pages(seq):
    """Neither taken nor given back, nor another sequence's in their place."""
    c = cache()
    c.reserve({0: 5, 2: 9})
    table, free = c.page_table.clone(), c.free_pages
    with pytest.raises(ValueError, match="sequence"):
        c.reserve({1: 4, seq: 9})
    with pytest.raises(ValueError, match="sequence"):
        c.release(seq)
    assert torch.equal(c.page_table, table) and c.free_pages == free
