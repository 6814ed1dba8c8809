"""A 4-bit head of a vocabulary that the bf16 GEMMs do not take, over more rows than one call takes."""
import math

import pytest
import torch

import adept_inputs as ai
from paper_2601_03700_amd import binding as B
from paper_2601_03700_amd.model import DecoderModel

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("family", ["llama", "gpt2"])
def test_all_rows_of_a_long_pass(family):
    """Every row against the same row in a call of at most 64.  The rows' norms are the same values;
    two f32 sums of k exact products are each within k 2^-23 of the sum of the magnitudes, which
    is at most |x| |w|."""
    n, T, D = 22, 970, 128
    kw = dict(n_layers=1, d_model=D, n_heads=2, head_dim=64, d_ff=128, vocab=50257)
    shape = (ai.DecoderShape(family="gpt2", max_pos=1024, **kw) if family == "gpt2"
             else ai.DecoderShape(**kw))
    w = (ai.gpt2_weights if family == "gpt2" else ai.decoder_weights)(shape, seed=2, dtype="bf16",
                                                                   std=0.05)
    m = DecoderModel(shape, w, dtype="bf16", rope_max_pos=1024, quant=True)
    assert n * T > B.quant_linear_max_rows(shape.vocab)
    print(f"4-bit head {family}: {n * T} rows", flush=True)
    res, _ = m.prefill(ai.token_ids(3, shape.vocab, n, T), B.exit_cfg(math.inf, 1), logits="all")
    assert res.logits.shape == (n * T, shape.vocab)
    gain, shift = (m.final_ln_g, m.final_ln_b) if m.gpt2 else (m.final_norm, None)
    x = math.sqrt(D) * float(gain.abs().max()) * (1 + 2.0 ** -7)
    if shift is not None:
        x += float(shift.float().norm()) * (1 + 2.0 ** -7)
    tol = 2 * (D + 2) * 2.0 ** -23 * x * m.lm_head.float().norm(dim=1)
    for i in range(0, n * T, 64):
        few = m._head(res.state, res.rows[i:i + 64])
        assert ((res.logits[i:i + 64] - few).abs() <= tol).all(), i     # (NaN is not)
