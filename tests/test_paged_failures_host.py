"""Forked and resized caches whose memory or copies fail, without a GPU: nothing is lost."""
import pytest
import torch

from paper_2601_03700_amd import binding as B
from paper_2601_03700_amd import model as M
from tests.test_paged_share_host import PAGE, cache, consistent, copies, own, read, write  # noqa: F401


def allocations_fail(monkeypatch, at):
    """From the at-th tensor on that a resize asks for (0: the first)."""
    left, empty = [at], torch.empty

    def fail(*args, **kw):
        if left[0] == 0:
            raise torch.OutOfMemoryError("no memory")
        left[0] -= 1
        return empty(*args, **kw)

    monkeypatch.setattr(M.torch, "empty", fail)


@pytest.mark.parametrize("kv,at", [("bf16", 0), ("bf16", 1), ("fp8", 0), ("fp8", 1), ("fp8", 2),
                                   ("fp8", 3)])
@pytest.mark.parametrize("n_pages", [20, 7])
def test_a_resize_without_memory_changes_nothing(monkeypatch, kv, at, n_pages):
    c = own(cache(n_pages=12, kv=kv))
    for b in range(4):
        write(c, b, 0, [10 * b + i for i in range(9)])
    c.release(1)
    c.release(2)
    want = {b: read(c, b, 9) for b in (0, 3)}
    before = (c.k, c.v, c.k_scale, c.v_scale, c.kv, c.page_table.clone(), c.free_pages)
    with monkeypatch.context() as m:
        allocations_fail(m, at)
        with pytest.raises(torch.OutOfMemoryError):
            c.resize(n_pages)
    for now, then in zip((c.k, c.v, c.k_scale, c.v_scale, c.kv), before):
        assert now is then
    assert torch.equal(c.page_table, before[5]) and c.free_pages == before[6] and c.n_pages == 12
    consistent(c)
    assert all(read(c, b, 9) == w for b, w in want.items())
    c.resize(n_pages)                               # and does it once there is memory
    own(c)
    consistent(c)
    assert c.n_pages == n_pages and c.kv.n_pages == n_pages + 1
    for t in (c.k, c.v, c.k_scale, c.v_scale):
        assert t is None or t.shape[1] == (n_pages + 1) * PAGE
    assert all(read(c, b, 9) == w for b, w in want.items())


@pytest.fixture
def no_copies(monkeypatch, copies):                        # noqa: F811
    def fail(*args, **kw):
        raise B.AdeptError("no copy")

    return lambda m: m.setattr(B, "paged_copy", fail)


def state(c):
    return ([list(p) for p in c._pages], list(c._users), list(c._free), c.shared_pages,
            c.page_table.tolist())


def test_a_copy_that_fails_takes_no_pages(monkeypatch, no_copies):
    c = own(cache())
    write(c, 0, 0, range(1, 11))
    c.fork(0, 2, 8)                                # two shared pages, seven free
    calls = [lambda: c.fork(0, [1, 3], 10),        # the open page for each
             lambda: c.reserve({2: 13}, 3),        # both shared pages, and two more
             lambda: c.reserve({0: 10, 2: 8}, 4)]  # of the first of the two
    for call in calls:
        then = state(c)
        with monkeypatch.context() as m:
            no_copies(m)
            with pytest.raises(B.AdeptError, match="no copy"):
                call()
        assert state(c) == then
        consistent(c)
    for call in calls:                             # and all of it is there for the next ones
        call()
        consistent(c)
    assert read(c, 0, 10) == read(c, 1, 10) == read(c, 3, 10) == list(range(1, 11))
    assert read(c, 2, 8) == list(range(1, 9))


def test_a_move_that_fails_moves_nothing(monkeypatch, no_copies):
    c = own(cache(n_pages=12))
    for b in range(4):
        write(c, b, 0, [10 * b + i for i in range(9)])
    c.release(0)
    for call in (c.compact, lambda: c.resize(9)):
        then = state(c), c.k, c.v, c.kv
        with monkeypatch.context() as m:
            no_copies(m)
            with pytest.raises(B.AdeptError, match="no copy"):
                call()
        assert state(c) == then[0] and (c.k is then[1] and c.v is then[2] and c.kv is then[3])
        assert all(read(c, b, 9) == [10 * b + i for i in range(9)] for b in (1, 2, 3))
        consistent(c)
