"""The workspace that adept_paged_attend asks for covers every call of fewer entries."""
import pytest

from paper_2601_03700_amd import binding as B

A = 1 << 20


@pytest.mark.parametrize("H,heads", [(32, 32), (4, 4), (64, 8), (25, 25), (40, 1)])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("dtype", [B.KV_BF16, B.KV_FP8])
def test_never_less_for_more(H, heads, hd, dtype):
    """In the entries, the sequences and the pages of a sequence: a bound of the entries that falls
    from call to call fits what was made for the first."""
    counts = [*range(0, 300), *range(300, 2100, 13), 4096, 9000, 70001, 1 << 20]
    pages = [1, 2, 3, 4, 5, 8, 64, 500, 70000]
    seqs = [1, 2, 3, 7, 200, 1024, 5000]
    kv = B.PagedKv(dtype, heads, hd, 64, 1 << 16, A, A, A, A)
    need = {(m, p, s): B.paged_attend_workspace_bytes(kv, H, m, s, p)
            for m in counts for p in pages for s in seqs}
    for (m, p, s), n in need.items():
        for more in ((counts[min(counts.index(m) + 1, len(counts) - 1)], p, s),
                     (m, pages[min(pages.index(p) + 1, len(pages) - 1)], s),
                     (m, p, seqs[min(seqs.index(s) + 1, len(seqs) - 1)])):
            assert need[more] >= n, ((m, p, s), more)
