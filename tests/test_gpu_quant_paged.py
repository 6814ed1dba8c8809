"""Drafted generation over 4-bit weights and a paged cache, in the model's type and in 8 bits: every
layer of every pass on the GPU's own inputs against the oracle with the quantised matrices, what the
cache holds, and the tokens against the logits that they come from."""
import math

import numpy as np
import pytest
import torch

import adept_inputs as ai
from oracle import adept_oracle as O
from paper_2601_03700_amd import binding as B
from paper_2601_03700_amd.model import DecoderModel
from tests import layer_check as LC
from tests.test_gpu_paged_model import Checker
from tests.test_gpu_quant_layers import GPT2, SMALL, weights

pytestmark = pytest.mark.gpu


class Check(Checker):
    """The attention over the pages and, in 8 bits, that they hold the pass's K and V quantised
    (Checker); q, K, V and the layer's output as layer_check.py has them (its bounds)."""

    def __init__(self, model, cache, held):
        super().__init__(model, cache)
        self.held, self.rep, self.exits, self.passes = held, LC.Report(), 0, 0

    def rows_of(self, t, i, st, rows):
        """K or V of a pass's rows at layer i, before an 8-bit cache rounds them."""
        if self.c.kv_dtype == "fp8":
            return LC.host((st.new_k if t == "k" else st.new_v)[i - 1][rows])
        return LC.host(getattr(self.c, t)[i - 1][st.slot[rows].long()])

    def __call__(self, i, st):
        super().__call__(i, st)
        s, cmp = self.m.shape, self.rep.check
        n = int(st.counts[(i - 1) & 1])
        if n == 0:
            return
        rows = st.active[(i - 1) & 1][:n].long()
        lw, pos = self.held["layers"][i - 1], st.pos[rows].cpu().numpy().astype(np.int64)
        hp, hc = LC.host(st.h[(i - 1) & 1][rows]), LC.host(st.h[i & 1][rows])
        k, v = O.layer_kv(lw, hp, pos, s)
        cmp(f"K (computed)@{i}", self.rows_of("k", i, st, rows), k, "bf16")
        cmp(f"V (computed)@{i}", self.rows_of("v", i, st, rows), v, "bf16")
        heads = lambda t: LC.host(t[:n]).reshape(n, s.n_heads, s.head_dim)
        cmp(f"q@{i}", heads(st.q_buf), O.layer_q(lw, s, hp, pos), "bf16")
        cmp(f"h (RMS-normalised)@{i}", LC.rms_rows(hc),
            LC.rms_rows(O.layer_out(lw, s, hp, heads(st.attn_out))), "bf16", allow=LC.RESID_ALLOW)

    def finish(self, res):
        """K and V of the layers that exited rows skipped, and the logits."""
        st, s = res.state, self.m.shape
        el = st.exit_layer.cpu().numpy().astype(np.int64)
        h = torch.where((st.exit_layer & 1).bool()[:, None], st.h[1], st.h[0])
        gone = np.nonzero(el < s.n_layers)[0]
        self.exits += gone.size
        self.passes += 1
        if gone.size:
            at = torch.from_numpy(gone).cuda()
            gen = O.kv_generate(self.held, s, LC.host(h[at]), el[gone],
                                st.pos[at].cpu().numpy().astype(np.int64))
            for r, (idx, k, v) in gen.items():
                rows = at[torch.from_numpy(np.asarray(idx)).cuda()]
                self.rep.check(f"K (generated)@{r}", self.rows_of("k", r, st, rows), k, "bf16")
                self.rep.check(f"V (generated)@{r}", self.rows_of("v", r, st, rows), v, "bf16")
        if res.logits is not None:
            want = O.lm_logits(self.held, s, LC.host(h[res.rows.long()]))
            self.rep.check("logits", LC.host(res.logits), want, "bf16", absolute=True)


@pytest.mark.parametrize("shape", [SMALL, GPT2], ids=["llama", "gpt2"])
@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("n,delta", [(1, math.inf), (3, math.inf), (3, 0.0)])
def test_drafted_generation(shape, kv, fused, n, delta):
    """Drafts leave at layer 2 of 3, the verifying passes never or by the policy.  Every token is
    the largest logit of the row of the token before it."""
    print(f"4-bit drafts {shape.family} {kv} fused={fused} {n} sequences, delta {delta}", flush=True)
    T, steps, g = 11, 10, 3
    w, held = weights(shape, 7)
    m = DecoderModel(shape, w, dtype="bf16", rope_max_pos=512, kv_fused=fused, quant=True)
    ids = ai.token_ids(n, shape.vocab, n, T)
    cache = m.new_paged_cache(n, n_pages=n * 4 + 2, page_size=8, kv_dtype=kv)
    for t in (cache.k, cache.v):         # what a pass does not write must not matter
        t.fill_(0x7f if kv == "fp8" else math.nan)
    check = Check(m, cache, held)
    said = {}                            # (sequence, position): the token there and the next one
    pass_of = m.token_pass

    def checked(ids, pos, seq, cache, cfg, force, tiles, rows):
        res = pass_of(ids, pos, seq, cache, cfg, force, tiles, rows, check)
        check.finish(res)
        if tiles:
            best = m.greedy(res.logits).tolist()
            for j, r in enumerate(res.rows.tolist()):
                said[int(seq[r]), int(pos[r])] = int(ids[r]), best[j]
        return res

    m.token_pass = lambda ids, pos, seq, cache, cfg, force=None, tiles=True, rows=None, on_layer=None: \
        checked(ids, pos, seq, cache, cfg, force, tiles, rows)
    out, kept, made, _ = m.generate_drafted(
        ids, steps, B.exit_cfg(delta, shape.n_layers, min_exit_layer=2),
        B.exit_cfg(-1.0, shape.n_layers, min_exit_layer=2), g, cache=cache)
    check.rep.summary()
    assert check.layers == shape.n_layers * check.passes and check.exits >= made // g
    assert 0 <= kept <= made
    out = out.tolist()
    for b in range(n):
        line = [int(ids[b][T - 1]), *out[b]]
        assert [said[b, T - 1 + t] for t in range(steps)] == list(zip(line, line[1:]))
