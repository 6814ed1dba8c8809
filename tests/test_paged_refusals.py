"""What the paged-cache entry points refuse, on the host: nothing is launched."""
import ctypes

import pytest
import torch

from paper_2601_03700_amd import binding as B
from tests.test_abi import test_struct_layout_matches_header as struct_layout

A = 1 << 20          # an aligned address that is never read


def kv(**change):
    d = dict(dtype=B.KV_BF16, n_kv_heads=2, head_dim=64, page_size=16, n_pages=8, k=A, v=A,
             k_scale=None, v_scale=None)
    d.update(change)
    return B.PagedKv(*(d[n] for n, _ in B.PagedKv._fields_))


def store(kv_, dt=B.BF16, k=A, ks=128, v=A, vs=128, n=4, slot=A):
    return B.lib().adept_paged_store(dt, ctypes.byref(kv_), k, ks, v, vs, None, None, n, slot, None)


def load(kv_, dt=B.BF16, k=A, ks=128, v=A, vs=128, n=4, slot=A):
    return B.lib().adept_paged_load(dt, ctypes.byref(kv_), slot, None, n, k, ks, v, vs, None)


def attend(kv_, dt=B.BF16, H=4, scale=0.125, causal=1, q=A, rows=A, n_active=A, n=3, pos=A, seq=A,
           n_seq=2, table=A, pages=4, key_len=None, out=A, ws=A, ws_bytes=1 << 40):
    return B.lib().adept_paged_attend(dt, ctypes.byref(kv_), H, scale, causal, q, rows, n_active, n,
                                      pos, seq, n_seq, table, pages, key_len, None, out, ws,
                                      ws_bytes, None)


def test_struct_layout(tmp_path):
    struct_layout(tmp_path, "adept_paged_kv", "PagedKv")


BAD_CACHES = [dict(dtype=3), dict(dtype=B.KV_F32), dict(n_kv_heads=0), dict(head_dim=96),
              dict(head_dim=8), dict(head_dim=512), dict(page_size=0), dict(page_size=24),
              dict(page_size=2048), dict(n_pages=0), dict(n_pages=1 << 27), dict(n_pages=(1 << 27) - 1), dict(k=None),
              dict(v=A + 8), dict(dtype=B.KV_FP8), dict(dtype=B.KV_FP8, k_scale=A),
              dict(dtype=B.KV_FP8, v_scale=A)]


@pytest.mark.parametrize("change", BAD_CACHES, ids=str)
@pytest.mark.parametrize("call", [store, load, attend])
def test_bad_caches(call, change):
    assert call(kv(**change)) == -1
    assert B.lib().adept_last_error()


@pytest.mark.parametrize("call", [store, load])
@pytest.mark.parametrize("bad", [dict(dt=2), dict(dt=B.F32), dict(k=None), dict(v=None),
                                 dict(slot=None), dict(k=A + 2), dict(v=A + 8), dict(ks=120),
                                 dict(vs=132), dict(n=-1), dict(n=(1 << 23) + 1)], ids=str)
def test_bad_rows(call, bad):
    assert call(kv(), **bad) == -1


@pytest.mark.parametrize("bad", [dict(dt=B.F32), dict(H=0), dict(H=3), dict(H=5000), dict(q=None),
                                 dict(rows=None), dict(n_active=None), dict(pos=None),
                                 dict(seq=None), dict(table=None), dict(out=None), dict(q=A + 4),
                                 dict(out=A + 8), dict(n=-1), dict(n=(1 << 23) + 1), dict(n_seq=0),
                                 dict(pages=0), dict(pages=1 << 27), dict(causal=0),
                                 dict(causal=2), dict(scale=0.0), dict(scale=float("inf")),
                                 dict(scale=float("nan")), dict(scale=-1.0)], ids=str)
def test_bad_attention(bad):
    assert attend(kv(), **bad) == -1


def test_missing_workspace():
    need = B.paged_attend_workspace_bytes(kv(), 4, 3, 2, 4)
    assert need > 0
    for bad in (dict(ws=None), dict(ws=A + 8), dict(ws_bytes=need - 1)):
        assert attend(kv(), **bad) == -3


def test_nothing_to_do_is_no_error():
    none = dict(k=None, v=None, slot=None, n=0)
    assert store(kv(), **none) == 0 and load(kv(), **none) == 0
    assert attend(kv(), n=0, q=None, rows=None, out=None) == 0


def t(*dims, dtype=torch.bfloat16):
    return torch.zeros(dims, dtype=dtype)


@pytest.mark.parametrize("args", [
    (t(32, 2, 64), t(32, 2, 64), 24),                               # slots no multiple of the page
    (t(32, 2, 64), t(32, 2, 32), 16), (t(32, 64), t(32, 64), 16),
    (t(32, 2, 64), t(32, 2, 64, dtype=torch.float32), 16),
    (t(32, 2, 64, dtype=torch.float16), t(32, 2, 64, dtype=torch.float16), 16),
    (t(2, 32, 64).transpose(0, 1), t(2, 32, 64).transpose(0, 1), 16),
    (t(32, 2, 64, dtype=torch.uint8), t(32, 2, 64, dtype=torch.uint8), 16),   # no scales
    (t(32, 2, 64), t(32, 2, 64), 16, t(32, 2, dtype=torch.uint8), t(32, 2, dtype=torch.uint8)),
    (t(32, 2, 64, dtype=torch.uint8), t(32, 2, 64, dtype=torch.uint8), 16,
     t(32, 2, dtype=torch.uint8), t(32, 2, 1, dtype=torch.uint8)),
])
def test_descriptor_checks(args):
    with pytest.raises(B.AdeptError):
        B.paged_kv(*args)


def test_tensors_elsewhere_are_refused():
    kv_ = B.paged_kv(t(32, 2, 64), t(32, 2, 64), 16)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(B.AdeptError, match="device"):
        B.paged_store(kv_, t(4, 2, 64), t(4, 2, 64), i)
    with pytest.raises(B.AdeptError, match="device"):
        B.paged_load(kv_, i, t(4, 2, 64), t(4, 2, 64))
    with pytest.raises(B.AdeptError, match="device"):
        B.paged_attend(kv_, t(4, 2, 64), i, i, 4, i, i, 1, i.view(1, 4), t(4, 2, 64))


@pytest.mark.parametrize("table,slots", [((2, 4), 5), ((3,), 5), ((3, 4), 4), ((3, 4), 5)])
def test_layer_step_checks_its_tables(table, slots):
    """Too few rows or slots; the last case fits and is refused for being on the host."""
    a = B.LayerArgs()
    a.n_seq, a.n_tok = 3, 5
    kv_ = B.paged_kv(t(8, 2, 64), t(8, 2, 64), 4)
    with pytest.raises(B.AdeptError, match="page_table|one slot|current HIP device"):
        B.layer_step_paged(a, kv_, t(*table, dtype=torch.int32), 1, t(slots, dtype=torch.int32))
