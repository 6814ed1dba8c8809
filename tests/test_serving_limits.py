"""Sizes that a call over 4-bit weights does not take: refused before anything is launched, and
what a model does with a pass of that many rows."""
import ctypes
from types import SimpleNamespace

import pytest
import torch

import adept_inputs as ai
from paper_2601_03700_amd import binding as B
from paper_2601_03700_amd.model import DecoderModel
from tests import test_serving_refusals as R

A = 1 << 20          # an aligned address that is never read


def head(vocab, rows):
    return B.lib().adept_final_logits_quant(256, vocab, 1e-6, A, A, A, A, A, rows, A, None, A, A, A, A,
                                            None)


@pytest.mark.parametrize("vocab,rows", [(100, -1), (100, 64 * 65535 + 1), (50257, 21297),
                                        (32000, 33425), (1 << 26, 16)])
def test_a_head_over_too_many_rows(vocab, rows):
    """The bound of the product, before the rows' norm."""
    assert head(vocab, rows) == -1
    assert b"final_logits_quant: bad max_rows" in B.lib().adept_last_error()


@pytest.mark.parametrize("n", [1, 16, 17, 321, 32000, 50257, 65521, 1 << 20])
def test_the_most_rows_of_a_call(n):
    """The sizes' check comes before the one of the tensors."""
    linear = lambda m: B.lib().adept_quant_linear(n, 64, None, 64, None, None, m, A, A, None, B.F32, None,
                                                  n, None)
    most = B.quant_linear_max_rows(n)
    assert most >= 16
    assert linear(most) == -1 and b"x must be" in B.lib().adept_last_error()
    assert linear(most + 1) == -1 and b"max_rows" in B.lib().adept_last_error()


@pytest.mark.parametrize("nr", [0, 1, 64, 65, 21296, 21297, 42592, 50000])
def test_a_head_that_no_call_takes_whole_is_split(monkeypatch, nr):
    """A vocabulary that the bf16 GEMMs do not take: passes of any size read the 4-bit head, in calls
    of the rows that one takes."""
    V, D, most = 50257, 8, 21296
    calls = []

    def head(d_model, vocab, eps, h0, h1, exit_layer, rows, n_rows, max_rows, gain, bias, qw, x_norm,
             logits):
        assert 0 < max_rows <= most == B.quant_linear_max_rows(vocab)
        assert rows.shape == (max_rows,) and n_rows.tolist() == [max_rows]
        assert x_norm.shape == (max_rows, D) and logits.shape == (max_rows, V)
        assert x_norm.is_contiguous() and logits.is_contiguous()
        calls.append((rows.tolist(), x_norm.storage_offset(), logits.storage_offset()))

    monkeypatch.setattr(B, "final_logits_quant", head)
    m = object.__new__(DecoderModel)
    m.shape = ai.DecoderShape(n_layers=1, d_model=D, n_heads=1, head_dim=8, d_ff=8, vocab=V)
    m.device, m.tdt, m.gpt2, m.final_norm = torch.device("cpu"), torch.bfloat16, False, None
    m.quant = {"lm_head": None}
    rows = torch.arange(nr, dtype=torch.int32).flip(0)
    logits = m._head(SimpleNamespace(h=[None, None], exit_layer=None), rows)
    assert logits.shape == (nr, V) and logits.dtype is torch.float32
    assert [r for c in calls for r in c[0]] == rows.tolist() and len(calls) == -(-nr // most)
    at = 0
    for r, x, y in calls:
        assert (x, y) == (at * D, at * V)
        at += len(r)


FP8 = dict(dtype=B.KV_FP8, k_scale=A, v_scale=A, n_kv_heads=4)


@pytest.mark.parametrize("a,c,table,pages,slot", [
    (dict(), dict(n_kv_heads=2), A, 4, None), (dict(), dict(n_kv_heads=4, page_size=3), A, 4, None),
    (dict(n_seq=0), dict(n_kv_heads=4), A, 4, None), (dict(), dict(n_kv_heads=4), None, 4, None),
    (dict(), dict(n_kv_heads=4), A, 4, None), (dict(), FP8, A, 4, None), (dict(n_slots=7), FP8, A, 4, A),
    (dict(k_cache=A + 2), FP8, A, 4, A), (dict(kv_fused=0, attn_tiles=0), FP8, A, 4, A)], ids=str)
def test_errors_of_paged_steps_name_the_call(a, c, table, pages, slot):
    args, cache = R.layer_args(**a), R.kv(**c)
    kv = ctypes.byref(cache)
    assert B.lib().adept_layer_step_quant(ctypes.byref(args), ctypes.byref(R.layer_weights()), kv, table,
                                          pages, slot, 1, None) == -1
    of_quant = B.lib().adept_last_error()
    assert of_quant.startswith(b"layer_step_quant: ")
    assert B.lib().adept_layer_step_paged(ctypes.byref(args), kv, table, pages, slot, 1, None) == -1
    assert B.lib().adept_last_error() == of_quant.replace(b"step_quant", b"step_paged")
