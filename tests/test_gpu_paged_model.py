"""DecoderModel over a PagedKVCache: prompts in pieces and decode passes, tokens exiting, in the
model's type and in 8 bits."""
import math

import numpy as np
import pytest
import torch

import adept_inputs as ai
from paper_2601_03700_amd import binding as B
from paper_2601_03700_amd.model import DecoderModel
from tests import paged_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"

LLAMA = ai.DecoderShape(n_layers=4, d_model=256, n_heads=4, head_dim=64, d_ff=512, vocab=128)
GPT2 = ai.DecoderShape(n_layers=3, d_model=256, n_heads=2, head_dim=128, d_ff=512, vocab=128,
                       family="gpt2", max_pos=256)


def build(shape, dtype, **kw):
    w = (ai.gpt2_weights if shape.family == "gpt2" else ai.decoder_weights)(shape, seed=3,
                                                                         dtype=dtype, std=0.04)
    return DecoderModel(shape, w, dtype=dtype, rope_max_pos=256, **kw)


class Checker:
    """After every layer: the attention of the rows that ran it, on the GPU's own q and on what
    the cache holds; in 8 bits also that the cache holds the pass's K and V, quantised."""

    def __init__(self, model, cache):
        self.m, self.c, self.worst, self.layers = model, cache, 0.0, 0

    def __call__(self, i, st):
        s, c = self.m.shape, self.c
        n = int(st.counts[(i - 1) & 1])
        rows = st.active[(i - 1) & 1][:n].long()
        k, v = c.k[i - 1], c.v[i - 1]
        if c.kv_dtype == "fp8":
            for new, codes, scale in ((st.new_k, k, c.k_scale[i - 1]), (st.new_v, v, c.v_scale[i - 1])):
                val, E = R.quantised(new[i - 1].cpu())
                at = st.cache_slot.long().cpu()
                assert torch.equal(R.cache_values(codes.cpu()[at], scale.cpu()[at]),
                                   val * R.power(E).unsqueeze(-1))
            k = R.cache_values(k.cpu(), c.k_scale[i - 1].cpu()).to(DEV)
            v = R.cache_values(v.cpu(), c.v_scale[i - 1].cpu()).to(DEV)
        q = st.q_buf.view(-1, s.n_heads, s.head_dim)[:n]
        ref, wv, qk = R.attend(q, k, v, c.page_table, c.page_size, st.pos[rows], st.seq[rows],
                               1 / math.sqrt(s.head_dim))
        err = (st.attn_out.view(-1, s.n_heads, s.head_dim)[:n].double() - ref).abs()
        assert torch.isfinite(ref).all()
        if n:
            self.worst = max(self.worst, (err / R.bound(q.dtype, ref, wv, qk)).max().item())
        assert self.worst <= 1.0
        self.layers += 1


def pieces(model, cache, ids, force, cuts, cfg, check):
    """The prompt in pieces that end at `cuts`: logits of all rows, in prompt order."""
    out, at = [], 0
    for end in cuts:
        res, _ = model.prefill(ids[:, at:end], cfg, force_layer=force[:, at:end], logits="all",
                               cache=cache, start=at, on_layer=check)
        out.append(res.logits.view(ids.shape[0], end - at, -1))
        at = end
    return torch.cat(out, 1)


CASES = [(LLAMA, "f32", "f32", 16), (LLAMA, "f32", "fp8", 8), (LLAMA, "bf16", "bf16", 4),
         (LLAMA, "bf16", "fp8", 64), (GPT2, "bf16", "bf16", 16), (GPT2, "bf16", "fp8", 16)]


@pytest.mark.parametrize("shape,dtype,kv,page", CASES)
@pytest.mark.parametrize("fused", [True, False])
def test_prompt_in_pieces_then_decode(shape, dtype, kv, page, fused):
    print(f"paged model {shape.family} {dtype}/{kv} page={page} fused={fused}", flush=True)
    n_seq, T, steps = 3, 90, 4
    model = build(shape, dtype, kv_fused=fused)
    ids = ai.token_ids(4, shape.vocab, n_seq, T)
    force = ai.forced_exit_layers(5, ids.size, 1, shape.n_layers).reshape(ids.shape)
    cfg = B.exit_cfg(math.inf, shape.n_layers)
    cache = model.new_paged_cache(n_seq, n_pages=n_seq * (-(-(T + steps) // page)) + 1,
                                  page_size=page, kv_dtype=kv)
    for t in (cache.k, cache.v):         # what a pass does not write must not matter
        t.fill_(0x7f if kv == "fp8" else math.nan)
    check = Checker(model, cache)
    logits = pieces(model, cache, ids, force, (37, 38, 80, T), cfg, check)
    nxt = model.greedy(logits[:, -1].contiguous())
    rng = np.random.default_rng(1)
    for j in range(steps):
        f = torch.from_numpy(rng.integers(0, shape.n_layers + 1, n_seq).astype(np.int32)).to(DEV)
        pos = torch.full((n_seq,), T + j, dtype=torch.int32, device=DEV)
        res = model.decode_step(cache, nxt, pos, cfg, force_layer=f, on_layer=check,
                                pos_max=T + j if j % 2 else None)
        assert torch.isfinite(res.logits).all()
        nxt = model.greedy(res.logits)
    assert check.layers == shape.n_layers * (4 + steps)
    # every layer holds finite K and V for every token of every sequence: generated and computed
    t = torch.arange(T + steps, dtype=torch.int32, device=DEV).repeat(n_seq)
    b = torch.arange(n_seq, dtype=torch.int32, device=DEV).repeat_interleave(T + steps)
    slot = cache.slots(t, b)
    for i in range(1, shape.n_layers + 1):
        k, v = (torch.empty((t.numel(), shape.n_heads, shape.head_dim), dtype=model.tdt, device=DEV)
                for _ in range(2))
        B.paged_load(cache.layer_kv(i), slot, k, v)
        assert torch.isfinite(k).all() and torch.isfinite(v).all()
    print(f"  worst error / bound {check.worst:.3f}", flush=True)


def test_same_as_over_the_contiguous_cache():
    """f32: the prompt in pieces over pages gives the logits, exits and cache of the whole prompt
    over a contiguous cache, to the rounding of f32 (1e-5 of the largest value, as for the
    oracle's parity), and so do the decode passes after it."""
    print("paged model, f32 against the contiguous cache", flush=True)
    shape, n_seq, T, steps = LLAMA, 2, 70, 3
    model = build(shape, "f32")
    ids = ai.token_ids(6, shape.vocab, n_seq, T)
    force = ai.forced_exit_layers(7, ids.size, 1, shape.n_layers).reshape(ids.shape)
    cfg = B.exit_cfg(math.inf, shape.n_layers)
    whole, flat = model.prefill(ids, cfg, s_max=T + steps, force_layer=force)
    cache = model.new_paged_cache(n_seq, n_pages=24, page_size=8)
    got = pieces(model, cache, ids, force, (1, 50, T), cfg, None)
    cont = model.new_cache(n_seq, T + steps)     # in pieces over the contiguous cache too
    also = pieces(model, cont, ids, force, (33, T), cfg, None)

    def close(a, b):
        assert (a - b).abs().max() <= 1e-5 * b.abs().max()

    ref = whole.logits.view(n_seq, T, -1)
    close(got, ref)
    close(also, ref)
    nxt = model.greedy(ref[:, -1].contiguous())
    for j in range(steps):
        pos = torch.full((n_seq,), T + j, dtype=torch.int32, device=DEV)
        f = torch.tensor([1 + j % shape.n_layers, 0], dtype=torch.int32, device=DEV)
        a = model.decode_step(cache, nxt, pos, cfg, force_layer=f)
        b = model.decode_step(flat, nxt, pos, cfg, force_layer=f)
        close(a.logits, b.logits)
        assert torch.equal(a.exit_layer, b.exit_layer)
        nxt = model.greedy(b.logits)
    t = torch.arange(T + steps, dtype=torch.int32, device=DEV).repeat(n_seq)
    b = torch.arange(n_seq, dtype=torch.int32, device=DEV).repeat_interleave(T + steps)
    at = cache.slots(t, b).long()
    for i in range(shape.n_layers):
        close(cache.k[i][at], flat.k[i])
        close(cache.v[i][at], flat.v[i])


def test_pages_of_finished_sequences_serve_new_ones():
    """A cache of few pages: a sequence is released, its pages go to another, whose results are
    those over a cache of its own."""
    print("paged model, pages used again", flush=True)
    shape = LLAMA
    model = build(shape, "bf16")
    cfg = B.exit_cfg(math.inf, shape.n_layers)
    a, b = (ai.token_ids(s, shape.vocab, 1, 60) for s in (8, 9))
    cache = model.new_paged_cache(1, n_pages=4, page_size=16)
    own = model.new_paged_cache(1, n_pages=9, page_size=16)
    model.prefill(a, cfg, cache=cache)
    with pytest.raises(ValueError):
        model.prefill(b, cfg, cache=cache, start=60)      # no pages for 120 tokens
    cache.release(0)
    got, _ = model.prefill(b, cfg, cache=cache, logits="all")
    want, _ = model.prefill(b, cfg, cache=own, logits="all")
    assert torch.equal(got.logits, want.logits)
    with pytest.raises(ValueError):
        model.prefill(np.concatenate([a, b]), cfg, cache=cache)     # more sequences
    with pytest.raises(ValueError):
        model.prefill(a, cfg, start=3)                                # nothing to continue
    with pytest.raises(ValueError):
        model.new_paged_cache(1, 4, kv_dtype="f32")


def test_layers_that_no_row_reaches_are_stored_too():
    """8 bits, every row gone after layer 1 and the caller's bound lowered to 0 from layer 2 on:
    each later layer still holds the generated K and V."""
    print("paged model, no row left, 8 bits", flush=True)
    shape, n_seq, T = LLAMA, 2, 20
    model = build(shape, "bf16")
    ids = torch.from_numpy(ai.token_ids(2, shape.vocab, n_seq, T)).to(DEV, torch.int32).view(-1)
    cache = model.new_paged_cache(n_seq, n_pages=8, page_size=8, kv_dtype="fp8")
    cache.reserve(T)
    n = ids.numel()
    pos = torch.arange(T, dtype=torch.int32, device=DEV).repeat(n_seq)
    seq = torch.arange(n_seq, dtype=torch.int32, device=DEV).repeat_interleave(T)
    force = torch.ones(n, dtype=torch.int32, device=DEV)
    st = model.new_state(n, pos, seq, cache.slots(pos, seq), force)
    B.embed(n, shape.d_model, shape.vocab, ids, model.embed, st.h[0])
    B.token_init(n, shape.n_layers, shape.d_model, st.active[0], st.counts, st.exit_layer, st.inertia)
    args = model.layer_args(st, cache, B.exit_cfg(math.inf, shape.n_layers), True)
    for i in range(1, shape.n_layers + 1):
        args.max_active = n if i == 1 else 0
        B.layer_step_paged(args, cache.kv, cache.page_table, i, st.cache_slot)
    assert (st.exit_layer == 1).all()
    at = st.cache_slot.long().cpu()
    for i in range(shape.n_layers):
        for new, codes, scale in ((st.new_k, cache.k, cache.k_scale), (st.new_v, cache.v, cache.v_scale)):
            val, E = R.quantised(new[i].cpu())
            assert torch.equal(R.cache_values(codes[i].cpu()[at], scale[i].cpu()[at]),
                               val * R.power(E).unsqueeze(-1))


def test_rows_without_a_page():
    """Rows beyond a sequence's pages: computed, and nothing of another sequence changes."""
    print("paged model, rows without a page", flush=True)
    shape = LLAMA
    model = build(shape, "bf16")
    cfg = B.exit_cfg(math.inf, shape.n_layers)
    cache = model.new_paged_cache(2, n_pages=6, page_size=8, max_pages=3)
    ids = ai.token_ids(3, shape.vocab, 2, 16)
    model.prefill(ids, cfg, cache=cache)
    k, v = cache.k.clone(), cache.v.clone()
    pos = torch.tensor([16, 23, 24, 1000, 3], dtype=torch.int32, device=DEV)
    seq = torch.tensor([0, 0, 0, 0, 1], dtype=torch.int32, device=DEV)
    model.token_pass(torch.full((5,), 7, dtype=torch.int32, device=DEV), pos.clamp(max=250), seq,
                     cache, cfg, None, True, torch.arange(5, device=DEV))
    own = int(cache.slots(pos[4:], seq[4:]))
    keep = torch.ones(cache.n_slots, dtype=torch.bool, device=DEV)
    keep[own] = keep[-1] = False
    for now, then in ((cache.k, k), (cache.v, v)):     # bits: slots not written yet may hold NaN
        assert torch.equal(now[:, keep].view(torch.int16), then[:, keep].view(torch.int16))


@pytest.mark.parametrize("metric", ["global", "local"])
def test_exits_by_the_policy_over_an_8_bit_cache(metric):
    """The policy's own exits (no schedule) in a prompt and decode passes over 8 bits."""
    print(f"paged model, policy {metric}, 8 bits", flush=True)
    shape = LLAMA
    model = build(shape, "bf16")
    ids = ai.token_ids(2, shape.vocab, 2, 64)
    sims = []
    model.prefill(ids, B.exit_cfg(math.inf, shape.n_layers, metric),
                  on_layer=lambda i, st: sims.append(st.sim_out.clone()) if i < shape.n_layers else None)
    s = torch.stack(sims)
    cfg = B.exit_cfg(float(s[torch.isfinite(s)].median()), shape.n_layers, metric)
    cache = model.new_paged_cache(2, n_pages=20, page_size=8, kv_dtype="fp8")
    check = Checker(model, cache)
    res, _ = model.prefill(ids, cfg, cache=cache, on_layer=check)
    el = res.exit_layer
    assert (el < shape.n_layers).any() and el.unique().numel() > 1     # rows leave one by one
    nxt = model.greedy(res.logits.view(2, 64, -1)[:, -1].contiguous())
    for j in range(3):
        pos = torch.full((2,), 64 + j, dtype=torch.int32, device=DEV)
        st = model.decode_step(cache, nxt, pos, cfg, on_layer=check)
        nxt = model.greedy(st.logits)
