"""Whole layers and the head over weights in 4 bits (adept_layer_step_quant,
adept_final_logits_quant): each layer on the GPU's own inputs against the oracle with the
quantised matrices (tests/layer_check.py), with exits, over both kinds of cache."""
import copy
import math
import sys

import numpy as np
import pytest
import torch

import adept_inputs as ai
from oracle import adept_oracle as O
from paper_2601_03700_amd import binding as B
from paper_2601_03700_amd.model import DecoderModel
from tests import layer_check as LC
from tests.quant_ref import quantised_fast

pytestmark = pytest.mark.gpu

# K of 6.5 pieces of 128 and 13; heads of 64 and 128; 16 and 32 weight rows of a workgroup
LLAMA = ai.DecoderShape(n_layers=3, d_model=832, n_heads=6, head_dim=128, d_ff=1664, vocab=384)
SMALL = ai.DecoderShape(n_layers=3, d_model=256, n_heads=4, head_dim=64, d_ff=640, vocab=321)
WIDE = ai.DecoderShape(n_layers=2, d_model=1472, n_heads=24, head_dim=128, d_ff=4352, vocab=8200)
GPT2 = ai.DecoderShape(n_layers=3, d_model=576, n_heads=9, head_dim=64, d_ff=1664, vocab=448,
                       family="gpt2", max_pos=512)


def weights(shape, seed):
    """(weights of the model, oracle weights with the matrices as 4 bits hold them); gains of one
    and no shifts, which the model folds into the matrices before it quantises them."""
    gpt2 = shape.family == "gpt2"
    w = (ai.gpt2_weights if gpt2 else ai.decoder_weights)(shape, seed=seed, dtype="bf16")
    for lw in w["layers"]:
        for k in lw:
            if k in ("attn_norm", "ffn_norm", "ln1_g", "ln2_g"):
                lw[k] = np.ones_like(lw[k])
            if k in ("ln1_b", "ln2_b"):
                lw[k] = np.zeros_like(lw[k])
    held = copy.deepcopy(w)
    for lw in held["layers"]:
        for k in lw:
            if np.ndim(lw[k]) == 2:
                lw[k] = quantised_fast(lw[k])
    head = "embed" if gpt2 else "lm_head"      # the checks read the embedding as the head only
    held[head] = quantised_fast(held[head])
    return w, O.as64(held)


def run(shape, seqs, rows, kv_fused=True, cache_kind=None):
    print(f"4-bit layers {shape.family} width={shape.d_model} {seqs}x{rows} fused={kv_fused} "
          f"cache={cache_kind}", flush=True)
    w, held = weights(shape, rows + seqs)
    model = DecoderModel(shape, w, dtype="bf16", rope_max_pos=512, kv_fused=kv_fused, quant=True)
    cfg = B.exit_cfg(math.inf, shape.n_layers)
    rng = np.random.default_rng(rows + seqs)
    ids = ai.token_ids(rows, shape.vocab, seqs, rows)
    force = rng.integers(0, shape.n_layers, size=ids.shape).astype(np.int32)
    rep = LC.Report(lambda *a: print(*a, file=sys.stderr, flush=True))
    cache = model.new_cache(seqs, rows + 1)
    check = lambda f: LC.DecoderLayerCheck(held, shape, cache, O.ExitConfig(delta=math.inf), "bf16",
                                           force_layer=f, report=rep)
    chk = check(force)
    B.timing_reset()
    B.timing_enable(True)
    res, _ = model.prefill(ids, cfg, force_layer=force, logits="all", cache=cache, on_layer=chk)
    chk.finish(res.state, res.logits, res.rows)
    f = rng.integers(0, shape.n_layers, size=seqs).astype(np.int32)
    chk = check(f)
    pos = torch.full((seqs,), rows, dtype=torch.int32, device="cuda")
    nxt = torch.from_numpy(ai.token_ids(seqs, shape.vocab, 1, seqs).reshape(-1).astype(np.int32)).cuda()
    r = model.decode_step(cache, nxt, pos, cfg, force_layer=torch.from_numpy(f).cuda(), on_layer=chk,
                          pos_max=rows)
    chk.finish(r.state, r.logits, r.rows)
    B.timing_enable(False)
    rep.summary()
    return B.timing_read()


@pytest.mark.parametrize("shape", [LLAMA, SMALL, GPT2], ids=["llama", "small", "gpt2"])
@pytest.mark.parametrize("seqs,rows", [(1, 1), (1, 17), (3, 5), (16, 2), (17, 1), (33, 1), (64, 1),
                                       (5, 15)])
def test_layers(shape, seqs, rows):
    run(shape, seqs, rows)


@pytest.mark.parametrize("seqs", [4, 20, 40])
def test_layers_of_32_weight_rows(seqs):
    run(WIDE, seqs, 1)


@pytest.mark.parametrize("shape", [SMALL, GPT2], ids=["small", "gpt2"])
def test_generation_after_the_layers(shape):
    run(shape, 6, 3, kv_fused=False)


def model_pair(shape, seed):
    """A model over 4 bits, and the bf16 one of the same matrices."""
    gpt2 = shape.family == "gpt2"
    m = DecoderModel(shape, (ai.gpt2_weights if gpt2 else ai.decoder_weights)(
        shape, seed=seed, dtype="bf16", std=0.04), rope_max_pos=512, quant=True)
    plain = copy.copy(m)
    plain.quant = plain._quant_struct = None
    return m, plain


@pytest.mark.parametrize("shape", [SMALL, GPT2], ids=["small", "gpt2"])
def test_larger_passes_are_those_of_the_unpacked_matrices(shape):
    if shape is SMALL:
        shape = ai.DecoderShape(n_layers=3, d_model=256, n_heads=4, head_dim=64, d_ff=640, vocab=320)
    m, plain = model_pair(shape, 5)
    ids = ai.token_ids(5, shape.vocab, 2, 50)
    cfg = B.exit_cfg(math.inf, shape.n_layers)
    a, _ = m.prefill(ids, cfg, logits="all")
    b, _ = plain.prefill(ids, cfg, logits="all")
    assert torch.equal(a.logits, b.logits)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("fused", [True, False])
def test_paged_caches(kv, fused):
    """The same layers over pages: a decode pass with exits as over the contiguous cache (bf16, bit
    for bit where the attention runs in the same order: one sequence), and finite over 8 bits."""
    m, _ = model_pair(SMALL, 6)
    m.kv_fused = fused
    ids = ai.token_ids(6, SMALL.vocab, 3, 20)
    cfg = B.exit_cfg(math.inf, SMALL.n_layers)
    force = np.array([2, 0, 1], np.int32)
    nxt = torch.tensor([3, 1, 7], dtype=torch.int32, device="cuda")
    pos = torch.full((3,), 20, dtype=torch.int32, device="cuda")
    out = []
    for cache in (m.new_cache(3, 32), m.new_paged_cache(3, 9, 8, kv_dtype=kv)):
        m.prefill(ids, cfg, logits=None, cache=cache)
        out.append(m.decode_step(cache, nxt, pos, cfg, force_layer=torch.from_numpy(force).cuda(),
                                 pos_max=20).logits)
    # f32 attention sums in another order and, in 8 bits, K and V within 2^-4 of their size
    scale = out[0].abs().max()
    assert torch.isfinite(out[1]).all()
    assert (out[0] - out[1]).abs().max() <= (2.0 ** -5 if kv == "bf16" else 2.0 ** -1) * scale


def test_refusals():
    w = ai.decoder_weights(SMALL, seed=1, dtype="f32")
    with pytest.raises(ValueError, match="bf16"):
        DecoderModel(SMALL, w, dtype="f32", quant=True)
    m, _ = model_pair(SMALL, 1)
    a = B.LayerArgs()
    a.n_layers, a.d_model, a.n_heads, a.head_dim, a.d_ff = 4, 256, 4, 64, 640
    with pytest.raises(B.AdeptError, match="4 matrices"):
        B.quant_layers(a, *(m.quant[n] for n in ("w_qkv", "w_o", "w_gate", "w_up", "w_down")))
