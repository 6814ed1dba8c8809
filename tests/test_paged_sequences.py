"""Sequences and lengths that a cache does not have, on the host."""
import pytest
import torch

from paper_2601_03700_amd.model import DecoderModel, KVCache, PagedKVCache


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


class Reached(Exception):
    pass


class HostModel(DecoderModel):
    """The checks before a pass, without the pass."""

    def __init__(self):
        self.device, self.rope_max_pos = torch.device("cpu"), 64

    def token_pass(self, *args):
        raise Reached


def flat(n_seq=2, s_max=8):
    k = torch.zeros((1, n_seq * s_max, 2, 16))
    return KVCache(k, k.clone(), n_seq, s_max)


@pytest.mark.parametrize("make", [flat, lambda: cache(n_seq=2, n_pages=4, page=4, max_pages=2)])
def test_passes_that_a_given_cache_cannot_hold(make):
    """More sequences or tokens than the cache has slots for would be written behind it."""
    m = HostModel()
    ids = lambda b, t: torch.zeros((b, t), dtype=torch.int32)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)
    for fits in (dict(ids=ids(2, 8)), dict(ids=ids(1, 3), start=5)):
        with pytest.raises(Reached):
            m.prefill(cfg=None, cache=make(), **fits)
    for bad in (dict(ids=ids(3, 4)), dict(ids=ids(3, 4), start=2), dict(ids=ids(2, 9)),
                dict(ids=ids(2, 9), s_max=9), dict(ids=ids(1, 4), start=5)):
        with pytest.raises(ValueError):
            m.prefill(cfg=None, cache=make(), **bad)
    with pytest.raises(Reached):
        m.decode_step(make(), i32(1, 1), i32(7, 0), None)
    for n, pos in ((3, i32(1, 1, 1)), (2, i32(8, 0))):
        with pytest.raises(ValueError):
            m.decode_step(make(), i32(*[1] * n), pos, None)
        with pytest.raises(ValueError):
            m.decode_step(make(), i32(*[1] * n), pos, None, pos_max=int(pos.max()))
