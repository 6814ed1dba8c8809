"""What draft verification, weights in 4 bits and page copies refuse, on the host: nothing is
launched."""
import ctypes

import pytest
import torch

from paper_2601_03700_amd import binding as B

A = 1 << 20          # an aligned address that is never read


def verify(dt=B.F32, n=2, g=3, V=100, target=A, ts=100, draft=A, ds=100, tokens=A, n_draft=None,
           temp=None, u=A, out=A, kept=A, ws=A, ws_bytes=1 << 40):
    return B.lib().adept_verify_drafts(dt, n, g, V, target, ts, draft, ds, tokens, n_draft, temp, u,
                                       out, kept, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [dict(dt=2), dict(n=-1), dict(g=-1), dict(V=0), dict(V=2**31 - 1),
                                 dict(n=1 << 20, g=1 << 10), dict(target=None), dict(u=None),
                                 dict(out=None), dict(kept=None), dict(tokens=None), dict(ts=99),
                                 dict(ds=99), dict(target=A + 2), dict(draft=A + 1),
                                 dict(dt=B.BF16, target=A + 1)], ids=str)
def test_verify_refuses(bad):
    assert verify(**bad) == -1
    assert B.lib().adept_last_error()


def test_verify_workspace():
    need = B.verify_drafts_workspace_bytes(2, 3, 100)
    assert need > 0
    assert verify(ws=None) == -3 and verify(ws_bytes=need - 1) == -3 and verify(ws=A + 8) == -3
    assert verify(n=0, target=None) == 0
    assert B.verify_drafts_workspace_bytes(0, 3, 100) == 0
    assert B.verify_drafts_workspace_bytes(2, -1, 100) == 0
    # what is made for a case serves every smaller one
    for smaller in ((1, 3, 100), (2, 2, 100), (2, 3, 7)):
        assert B.verify_drafts_workspace_bytes(*smaller) <= need


def pack(dt=B.BF16, n=20, k=40, w=A, ldw=40, codes=A, scales=A):
    return B.lib().adept_quant_pack(dt, n, k, w, ldw, codes, scales, None)


def unpack(dt=B.BF16, n=20, k=40, w=A, ldw=40, codes=A, scales=A):
    return B.lib().adept_quant_unpack(dt, n, k, codes, scales, w, ldw, None)


@pytest.mark.parametrize("call", [pack, unpack])
@pytest.mark.parametrize("bad", [dict(dt=2), dict(n=0), dict(k=0), dict(n=2**31 - 1), dict(w=None),
                                 dict(ldw=39), dict(codes=None), dict(scales=None), dict(codes=A + 8),
                                 dict(scales=A + 4), dict(w=A + 1), dict(n=1 << 30, k=1 << 10, ldw=1 << 10),
                                 dict(k=(1 << 29) + 8, ldw=1 << 30)],
                         ids=str)
def test_pack_refuses(call, bad):
    assert call(**bad) == -1


def linear(n=20, k=40, x=A, xs=40, rows=None, n_rows=None, m=3, codes=A, scales=A, bias=None,
           dt=B.F32, y=A, ys=20):
    return B.lib().adept_quant_linear(n, k, x, xs, rows, n_rows, m, codes, scales, bias, dt, y, ys,
                                      None)


@pytest.mark.parametrize("bad", [dict(n=0), dict(k=0), dict(k=44, xs=48), dict(x=None), dict(x=A + 8),
                                 dict(xs=32), dict(xs=44), dict(m=-1), dict(m=64 * 65536), dict(n=32000, ys=32000, m=33600),
                                 dict(codes=None), dict(scales=A + 8), dict(bias=A + 1), dict(dt=2),
                                 dict(y=None), dict(ys=19), dict(y=A + 2),
                                 dict(dt=B.BF16, y=A + 1)], ids=str)
def test_linear_refuses(bad):
    assert linear(**bad) == -1
    assert B.lib().adept_last_error()


def test_no_rows_is_no_call():
    assert linear(m=0, x=None, y=None) == 0


def test_sizes():
    L = B.lib()
    assert L.adept_quant_codes_bytes(16, 128) == 1024 and L.adept_quant_scales_bytes(16, 128) == 64
    assert L.adept_quant_codes_bytes(17, 129) == 4096 and L.adept_quant_scales_bytes(1, 1) == 64
    assert L.adept_quant_codes_bytes(0, 5) == 0 and L.adept_quant_scales_bytes(5, -1) == 0
    assert L.adept_quant_codes_bytes(1 << 20, 1 << 14) == 1 << 33


def kv(**change):
    d = dict(dtype=B.KV_BF16, n_kv_heads=2, head_dim=64, page_size=16, n_pages=8, k=A, v=A,
             k_scale=None, v_scale=None)
    d.update(change)
    return B.PagedKv(*(d[n] for n, _ in B.PagedKv._fields_))


def copy(kv_=None, layers=2, src=A, dst=A, n=3):
    kv_ = kv() if kv_ is None else kv_
    return B.lib().adept_paged_copy(ctypes.byref(kv_), layers, src, dst, None, None, n, None)


@pytest.mark.parametrize("change", [dict(dtype=3), dict(n_kv_heads=0), dict(head_dim=96),
                                    dict(page_size=24), dict(n_pages=0), dict(k=None), dict(v=A + 8),
                                    dict(dtype=B.KV_FP8)], ids=str)
def test_copy_refuses_bad_caches(change):
    assert copy(kv(**change)) == -1


@pytest.mark.parametrize("bad", [dict(layers=0), dict(src=None), dict(dst=None), dict(n=-1),
                                 dict(n=1 << 24)], ids=str)
def test_copy_refuses(bad):
    assert copy(**bad) == -1
    assert B.lib().adept_paged_copy(None, 1, A, A, None, None, 1, None) == -1
    assert copy(n=0, src=None) == 0


def test_the_binding_refuses_tensors_that_do_not_fit():
    t = torch.zeros((2, 4, 10))
    with pytest.raises(B.AdeptError, match="device"):
        B.verify_drafts(t, None, torch.zeros((2, 3), dtype=torch.int32), t[:, :, 0], None, None)
    with pytest.raises(B.AdeptError, match="no matrix"):
        B.quant_weights(0, 8, "cpu")
    with pytest.raises(B.AdeptError, match="no matrix"):
        B.quant_weights(8, 8, "cpu", 0)
    qw = B.quant_weights(16, 128, "cpu")
    for call in (lambda: B.quant_pack(torch.zeros(16, 128), qw),
                 lambda: B.quant_linear(torch.zeros((1, 128), dtype=torch.bfloat16), qw,
                                        torch.zeros(1, 16))):
        with pytest.raises(B.AdeptError, match="device"):
            call()
    with pytest.raises(B.AdeptError, match="distance"):
        B._logit_rows("x", torch.zeros(2, 4, 12)[:, :3, :10], 2, 3, 10)
    assert B._logit_rows("x", torch.zeros(2, 3, 12)[:, :, :10], 2, 3, 10) == 12
    assert B._logit_rows("x", torch.zeros(2, 4, 10)[:, :1], 2, 1, 10) == 40


def layer_args(**change):
    a = B.LayerArgs()
    for name, kind in B.LayerArgs._fields_:
        if kind is ctypes.c_void_p:
            setattr(a, name, A)
    a.dtype, a.n_layers, a.d_model, a.n_heads, a.head_dim, a.d_ff = B.BF16, 4, 256, 4, 64, 512
    a.family, a.rms_eps, a.exit = 0, 1e-6, B.exit_cfg(0.9, 4)
    a.n_tok = a.max_active = a.n_seq = a.n_slots = 8
    a.s_max = a.rope_max_pos = 1
    a.hsm = None
    a.active[0], a.active[1], a.n_active[0], a.n_active[1] = A, 2 * A, A, 2 * A
    a.h[0], a.h[1] = A, 2 * A
    a.workspace_bytes = 1 << 40
    for k, v in change.items():
        setattr(a, k, v)
    return a


def layer_weights(**change):
    w = B.QuantLayers()
    for name, _ in B.QuantLayers._fields_:
        setattr(w, name, change.get(name, B.QuantMat(A, A)))
    return w


def step(a, w, kv_=None, table=None, pages=0, layer=1):
    ref = lambda x: None if x is None else ctypes.byref(x)
    return B.lib().adept_layer_step_quant(ref(a), ref(w), ref(kv_), table, pages, None, layer, None)


def test_layer_steps_refuse():
    assert step(None, layer_weights()) == -1 and step(layer_args(), None) == -1
    assert step(layer_args(dtype=B.F32), layer_weights()) == -1
    for name in ("qkv", "o", "gate", "up", "down"):
        for bad in (B.QuantMat(None, A), B.QuantMat(A, None), B.QuantMat(A + 8, A), B.QuantMat(A, A + 4)):
            assert step(layer_args(), layer_weights(**{name: bad})) == -1, name
            assert b"codes and scales" in B.lib().adept_last_error()
    assert step(layer_args(), layer_weights(), layer=5) == -1
    # the GPT2 family has no second projection of that kind
    assert step(layer_args(family=B.FAMILY_GPT2, d_ff=100), layer_weights(up=B.QuantMat())) == -1
    assert b"codes and scales" not in B.lib().adept_last_error()
    # over pages: the checks of the paged step
    assert step(layer_args(), layer_weights(), kv(n_kv_heads=2)) == -1
    assert b"heads" in B.lib().adept_last_error()
    assert step(layer_args(), layer_weights(), kv(n_kv_heads=4), None, 4) == -1
    assert b"page table" in B.lib().adept_last_error()
    need = B.lib().adept_layer_quant_workspace_bytes(ctypes.byref(layer_args()),
                                                     ctypes.byref(layer_weights()), None, 0)
    assert need > 0
    assert step(layer_args(workspace_bytes=need - 1), layer_weights()) == -3
    assert B.lib().adept_layer_quant_workspace_bytes(None, None, None, 0) == 0


def test_heads_refuse():
    f = B.lib().adept_final_logits_quant
    good = [256, 100, 1e-6, A, A, A, A, A, 4, A, None, A, A, A, A, None]
    for i, bad in ((0, 252), (0, 0), (1, 0), (3, None), (4, None), (5, None), (6, None), (8, -1),
                   (9, None), (11, None), (12, A + 8), (13, None), (14, A + 8), (10, A + 2), (3, A + 8)):
        args = list(good)
        args[i] = bad
        assert f(*args) == -1, (i, bad)
    args = list(good)
    args[8] = 0
    assert f(*args) == 0
