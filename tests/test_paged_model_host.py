"""The page bookkeeping of PagedKVCache and the checks of adept_layer_step_paged, without a GPU."""
import ctypes

import pytest
import torch

from paper_2601_03700_amd import binding as B
from paper_2601_03700_amd.model import PagedKVCache

A = 1 << 20


def cache(n_seq=3, n_pages=6, page=4, max_pages=4, kv="bf16"):
    return PagedKVCache(2, 2, 16, n_seq, n_pages, page, max_pages, kv, "cpu")


def test_pages_are_taken_as_sequences_grow_and_given_back():
    c = cache()
    assert (c.n_slots, c.s_max, c.free_pages) == (28, 16, 6)    # a page more, for no one
    c.reserve({0: 5, 2: 1})
    assert c.free_pages == 3 and (c.page_table >= 0).sum(1).tolist() == [2, 0, 1]
    c.reserve({0: 8})                      # fits the pages it has
    assert c.free_pages == 3
    c.reserve({0: 9, 1: 4})
    used = c.page_table[c.page_table >= 0].tolist()
    assert sorted(used) == sorted(set(used)) and len(used) == 5
    with pytest.raises(ValueError, match="free"):
        c.reserve({1: 9, 2: 5})
    assert c.free_pages == 1               # nothing was taken
    c.release(0)
    assert c.free_pages == 4 and (c.page_table[0] == -1).all()
    c.reserve({1: 9, 2: 5})
    with pytest.raises(ValueError, match="up to 16"):
        c.reserve({1: 17})
    c.release(0)                           # has none
    used = c.page_table[c.page_table >= 0].tolist()
    assert len(used) == len(set(used)) == 6 - c.free_pages


def test_slots():
    c = cache(page=4)
    c.reserve({0: 6, 1: 3})
    pos = torch.tensor([0, 5, 2, 7, 9, 16, -1], dtype=torch.int32)
    seq = torch.tensor([0, 0, 1, 1, 2, 0, 0], dtype=torch.int32)
    t = c.page_table
    want = [int(t[0, 0]) * 4, int(t[0, 1]) * 4 + 1, int(t[1, 0]) * 4 + 2] + [27] * 4
    got = c.slots(pos, seq)
    assert got.dtype == torch.int32 and got.tolist() == want


def test_layers_lie_behind_each_other():
    for kv in ("bf16", "f32", "fp8"):
        c = cache(kv=kv)
        first, second = c.layer_kv(1), c.layer_kv(2)
        e = c.k.element_size()
        assert second.k - first.k == c.n_slots * 2 * 16 * e == second.v - first.v
        assert first.n_pages == 7 and first.dtype == {"f32": 0, "bf16": 1, "fp8": 2}[kv]
        if kv == "fp8":
            assert second.k_scale - first.k_scale == c.n_slots * 2


def args(**change):
    a = B.LayerArgs()
    for name, kind in B.LayerArgs._fields_:
        if kind is ctypes.c_void_p:
            setattr(a, name, A)
    a.dtype, a.n_layers, a.d_model, a.n_heads, a.head_dim, a.d_ff = B.BF16, 4, 256, 4, 64, 512
    a.family, a.rms_eps, a.exit = 0, 1e-6, B.exit_cfg(0.9, 4)
    a.n_tok = a.max_active = a.n_seq = 8
    a.n_slots, a.s_max, a.rope_max_pos = 128, 1, 64
    a.kv_fused, a.attn_tiles, a.hsm = 1, 0, None
    a.active[0] = a.active[1] = a.n_active[0] = a.n_active[1] = a.h[0] = a.h[1] = A
    a.workspace, a.workspace_bytes = A, 1 << 40
    for k, v in change.items():
        setattr(a, k, v)
    return a


def kv(**change):
    d = dict(dtype=B.KV_BF16, n_kv_heads=4, head_dim=64, page_size=16, n_pages=8, k=A, v=A,
             k_scale=None, v_scale=None)
    d.update(change)
    return B.PagedKv(*(d[n] for n, _ in B.PagedKv._fields_))


FP8 = dict(dtype=B.KV_FP8, k_scale=A, v_scale=A)


@pytest.mark.parametrize("a,c,table,pages,slot", [
    (dict(), dict(n_kv_heads=2), A, 4, None), (dict(), dict(head_dim=128), A, 4, None),
    (dict(), dict(k=2 * A), A, 4, None), (dict(), dict(v=2 * A), A, 4, None),
    (dict(n_slots=64), dict(), A, 4, None), (dict(), dict(), None, 4, None),
    (dict(), dict(), A, 0, None), (dict(), dict(), A, 1 << 27, None),
    (dict(), dict(dtype=B.KV_F32), A, 4, None), (dict(), FP8, A, 4, None),
    (dict(kv_fused=0), FP8, A, 4, A), (dict(n_slots=7), FP8, A, 4, A),
    (dict(k_cache=A + 2), FP8, A, 4, A), (dict(n_tok=(1 << 23) + 1), dict(), A, 4, None),
    (dict(n_seq=0), dict(), A, 4, None), (dict(n_layers=0), dict(), A, 4, None)], ids=str)
def test_layer_step_refusals(a, c, table, pages, slot):
    status = B.lib().adept_layer_step_paged(ctypes.byref(args(**a)), ctypes.byref(kv(**c)), table,
                                            pages, slot, 1, None)
    assert status == -1 and B.lib().adept_last_error()


def test_layer_step_needs_its_workspace():
    a, c = args(), kv()
    need = B.lib().adept_layer_paged_workspace_bytes(ctypes.byref(a), ctypes.byref(c), 4)
    assert need > B.lib().adept_paged_attend_workspace_bytes(ctypes.byref(c), 4, 8, 8, 4) > 0
    a.workspace_bytes = need - 1
    assert B.lib().adept_layer_step_paged(ctypes.byref(a), ctypes.byref(c), A, 4, None, 1, None) == -3
    assert B.lib().adept_layer_step_paged(None, ctypes.byref(c), A, 4, None, 1, None) == -1
    assert B.lib().adept_layer_step_paged(ctypes.byref(a), None, A, 4, None, 1, None) == -1
