"""Arguments that the paged binding refuses before it looks for a device."""
import pytest
import torch

from paper_2601_03700_amd import binding as B


def t(*dims, dtype=torch.bfloat16):
    return torch.zeros(dims, dtype=dtype)


KV = B.paged_kv(t(32, 2, 64), t(32, 2, 64), 16)
I32 = torch.zeros(4, dtype=torch.int32)


@pytest.fixture(autouse=True)
def on_the_current_device(monkeypatch):
    """The host stands for the device; nothing of a good call is launched here."""
    monkeypatch.setattr(B, "_device_of", lambda what, kv: -1)


@pytest.mark.parametrize("dims", [(4, 128), (4,), (1, 4, 2, 64)])
def test_queries_that_have_no_heads(dims):
    with pytest.raises(B.AdeptError, match="q and out"):
        B.paged_attend(KV, t(*dims), I32, I32, 4, I32, I32, 1, I32.view(1, 4), t(*dims))


@pytest.mark.parametrize("call", [
    lambda n: B.paged_store(KV, t(4, 2, 64), t(4, 2, 64), I32, n_rows=n),
    lambda n: B.paged_store(KV, t(4, 2, 64), t(4, 2, 64), I32, rows=I32, n_rows=n),
    lambda n: B.paged_load(KV, I32, t(4, 2, 64), t(4, 2, 64), n_rows=n)])
def test_a_count_of_no_elements(call):
    """Its address is NULL, which would stand for all rows."""
    with pytest.raises(B.AdeptError, match="n_rows"):
        call(I32[:0])
