"""Page bookkeeping of forked, truncated, compacted and resized caches, without a GPU: what the
pages hold is followed through a copy in torch."""
import numpy as np
import pytest
import torch

from paper_2601_03700_amd import binding as B
from paper_2601_03700_amd.model import PagedKVCache

PAGE = 4


def cache(n_seq=4, n_pages=10, max_pages=5, kv="bf16"):
    return PagedKVCache(2, 2, 16, n_seq, n_pages, PAGE, max_pages, kv, "cpu")


@pytest.fixture(autouse=True)
def copies(monkeypatch):
    """binding.paged_copy by torch; the copied (source, destination, tokens)."""
    seen = []

    def copy(kv, n_layers, src, dst, n_tokens=None, n_pages=None, stream=None):
        assert len(set(dst.tolist())) == len(dst) and not set(dst.tolist()) & set(src.tolist())
        base = kv.owner
        for i, (s, d) in enumerate(zip(src.tolist(), dst.tolist())):
            m = PAGE if n_tokens is None else int(n_tokens[i])
            seen.append((s, d, m))
            for t in (base.k, base.v):
                t[:n_layers, d * PAGE:d * PAGE + m] = t[:n_layers, s * PAGE:s * PAGE + m]

    monkeypatch.setattr(B, "paged_copy", copy)
    return seen


def own(c):
    c.kv.owner = c
    return c


def write(c, seq, start, values):
    """Tokens of a sequence as a pass writes them."""
    c.reserve({seq: start + len(values)}, start)
    pos = torch.arange(start, start + len(values), dtype=torch.int32)
    at = c.slots(pos, torch.full_like(pos, seq)).long()
    for t in (c.k, c.v):
        t[:, at] = torch.tensor(values, dtype=t.dtype)[None, :, None, None].expand(2, -1, 2, 16)


def read(c, seq, n):
    pos = torch.arange(n, dtype=torch.int32)
    at = c.slots(pos, torch.full_like(pos, seq)).long()
    x = c.k[:, at]
    assert (x == x[:1, :, :1, :1]).all() and torch.equal(x, c.v[:, at])
    return x[0, :, 0, 0].tolist()


def consistent(c):
    """Users, free list and table say the same."""
    users = [0] * c.n_pages
    for b, pages in enumerate(c._pages):
        for p in pages:
            users[p] += 1
        row = c.page_table[b].tolist()
        assert row == pages + [-1] * (c.max_pages - len(pages))
    assert users == c._users
    assert sorted(c._free) == [p for p in range(c.n_pages) if users[p] == 0]
    assert c.shared_pages == sum(u > 1 for u in users)


def test_forks_share_full_pages_and_copy_the_open_one(copies):
    c = own(cache())
    write(c, 0, 0, range(1, 11))                   # 2 full pages and 2 tokens
    c.fork(0, [1, 3], 10)
    consistent(c)
    assert [m for _, _, m in copies] == [2, 2] and c.shared_pages == 2 and c.free_pages == 5
    write(c, 0, 10, [50, 51, 52])
    write(c, 1, 10, [60])
    write(c, 3, 10, [70, 71])
    assert read(c, 0, 13) == [*range(1, 11), 50, 51, 52]
    assert read(c, 1, 11) == [*range(1, 11), 60] and read(c, 3, 12) == [*range(1, 11), 70, 71]
    consistent(c)
    c.release(0)
    assert c.shared_pages == 2 and read(c, 1, 11) == [*range(1, 11), 60]
    c.fork(3, 0, 8)                                # whole pages: nothing copied
    assert len(copies) == 2 and c.shared_pages == 2
    c.fork(1, np.int64(2), 0)                      # of nothing
    consistent(c)
    for b in range(4):
        c.release(b)
    assert c.free_pages == 10
    consistent(c)


def test_a_write_into_a_shared_page_copies_it_first(copies):
    c = own(cache())
    write(c, 0, 0, range(1, 13))
    c.fork(0, [1, 2], 12)
    assert not copies
    write(c, 1, 6, [90, 91])                       # the second page of sequence 1
    assert read(c, 1, 12) == [1, 2, 3, 4, 5, 6, 90, 91, 9, 10, 11, 12]
    assert read(c, 0, 12) == read(c, 2, 12) == list(range(1, 13))
    consistent(c)
    # two of the remaining users at once: one copy is enough
    n = len(copies)
    c.reserve({0: 8, 2: 8}, {0: 4, 2: 7})
    assert len(copies) == n + 1
    consistent(c)
    c.reserve({0: 12})                             # no start: appended to
    assert len(copies) == n + 1
    c.fork(1, 3, 8)
    c.reserve({1: 12, 3: 12}, {3: 4})              # of one of them only
    assert len(copies) == n + 2 and copies[-1][0] == c._pages[1][1]
    consistent(c)


def test_nothing_is_taken_where_copies_do_not_fit(copies):
    c = own(cache(n_pages=4))
    write(c, 0, 0, range(1, 13))
    c.fork(0, 1, 12)
    with pytest.raises(ValueError, match="3 more pages needed, 1 free"):
        c.reserve({1: 12}, 0)
    with pytest.raises(ValueError, match="2 more pages needed"):
        c.reserve({1: 16}, 8)
    consistent(c)
    assert c.free_pages == 1 and not copies
    c.release(1)
    with pytest.raises(ValueError, match="2 more pages needed, 1 free"):
        c.fork(0, [1, 2], 6)
    consistent(c)
    assert c.free_pages == 1


@pytest.mark.parametrize("src,dst,length", [(0, 0, 4), (0, [1, 1], 4), (0, 2, 4), (0, 1, 13),
                                            (0, 1, -1), (0, 9, 4), (7, 1, 4), (0, -1, 4)])
def test_forks_that_are_refused(src, dst, length):
    c = own(cache())
    write(c, 0, 0, range(12))
    write(c, 2, 0, [1])
    with pytest.raises(ValueError):
        c.fork(src, dst, length)
    consistent(c)


def test_truncated_sequences_grow_again():
    c = own(cache())
    write(c, 0, 0, range(1, 14))
    c.truncate(0, 6)
    assert c.free_pages == 8 and read(c, 0, 6) == [1, 2, 3, 4, 5, 6]
    c.truncate(0, 6)
    c.truncate(0, 100)                             # has no more than that
    consistent(c)
    write(c, 0, 6, [7, 8, 9])
    assert read(c, 0, 9) == list(range(1, 10))
    with pytest.raises(ValueError):
        c.truncate(0, -1)
    with pytest.raises(ValueError, match="sequence 4"):
        c.truncate(4, 0)
    # a fork that goes back into a shared page
    c.fork(0, 1, 9)
    c.truncate(1, 3)
    write(c, 1, 3, [40])
    assert read(c, 0, 9) == list(range(1, 10)) and read(c, 1, 4) == [1, 2, 3, 40]
    consistent(c)


def test_compacted_and_resized(copies):
    c = own(cache(n_pages=12))
    for b in range(4):
        write(c, b, 0, [10 * b + i for i in range(9)])
    c.release(1)
    c.fork(3, 1, 8)
    want = {b: read(c, b, n) for b, n in ((0, 9), (1, 8), (2, 9), (3, 9))}
    same = lambda: all(read(c, b, len(w)) == w for b, w in want.items())
    c.release(0)
    del want[0]
    used = c.n_pages - c.free_pages
    assert used == 6 and c.compact() == len(copies) > 0
    consistent(c)
    assert int(c.page_table.max()) == used - 1 and same()
    assert c.compact() == 0
    c.resize(used)
    own(c)
    consistent(c)
    assert c.n_pages == used and c.free_pages == 0 and c.n_slots == (used + 1) * PAGE and same()
    with pytest.raises(ValueError, match="in use"):
        c.resize(used - 1)
    c.resize(20)
    own(c)
    consistent(c)
    assert c.free_pages == 14 and same()
    write(c, 0, 0, range(20))
    assert read(c, 0, 20) == list(range(20)) and same()
    c.release(0)
    write(c, 2, 9, [99])
    c.resize(8)                                    # moves what lies behind, if anything does
    own(c)
    consistent(c)
    want[2].append(99)
    assert same()
    with pytest.raises(ValueError):
        c.resize(0)


def test_an_empty_cache_is_moved_and_resized():
    c = own(cache())
    assert c.compact() == 0
    c.resize(3)
    consistent(own(c))
    c.reserve({0: 12})
    consistent(c)
