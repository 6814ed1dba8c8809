"""Drafted generation: draft passes that leave early, one pass that verifies them, over both kinds
of cache; sequences that fork, shrink and move in a paged one."""
import math

import numpy as np
import pytest
import torch

import adept_inputs as ai
from paper_2601_03700_amd import binding as B
from paper_2601_03700_amd.model import DecoderModel
from tests.verify_ref import verify

pytestmark = pytest.mark.gpu
SHAPE = ai.DecoderShape(n_layers=4, d_model=256, n_heads=4, head_dim=64, d_ff=512, vocab=320)
GPT2 = ai.DecoderShape(n_layers=3, d_model=256, n_heads=2, head_dim=128, d_ff=512, vocab=320,
                       family="gpt2", max_pos=256)
INF = math.inf


def build(dtype="f32", shape=SHAPE, **kw):
    w = (ai.gpt2_weights if shape.family == "gpt2" else ai.decoder_weights)(
        shape, seed=3, dtype=dtype, std=0.05)
    return DecoderModel(shape, w, dtype=dtype, rope_max_pos=256, **kw)


def never(shape=SHAPE):
    return B.exit_cfg(INF, shape.n_layers)


def early(shape=SHAPE, delta=0.5):
    return B.exit_cfg(delta, shape.n_layers, min_exit_layer=1)


@pytest.mark.parametrize("dtype,shape,kv,quant", [
    ("f32", SHAPE, None, False), ("bf16", SHAPE, None, False), ("bf16", GPT2, None, False),
    ("bf16", SHAPE, None, True), ("f32", SHAPE, "f32", False), ("bf16", SHAPE, "bf16", False),
    ("bf16", GPT2, "fp8", False), ("bf16", SHAPE, "fp8", True)])
@pytest.mark.parametrize("n,g", [(1, 4), (5, 3)])
def test_greedy_tokens_are_the_models(dtype, shape, kv, quant, n, g):
    """Every token is the largest logit of one pass over the whole sequence, up to the passes'
    rounding: f32 1e-3, bf16 twice the 2e-2 that a pass's logits are held to; an 8-bit cache
    rounds K and V themselves, and only its counts are held."""
    m = build(dtype, shape, **(dict(quant=True) if quant else {}))
    T, steps = 11, 17
    ids = ai.token_ids(7, shape.vocab, n, T)
    cache = None if kv is None else m.new_paged_cache(n, n * 5, 8, kv_dtype=kv)
    out, kept, made, cache = m.generate_drafted(ids, steps, never(shape), early(shape), g,
                                                cache=cache)
    assert out.shape == (n, steps) and 0 <= kept <= made and made % g == 0
    assert ((out >= 0) & (out < shape.vocab)).all()
    if kv == "fp8":
        return
    whole = torch.cat([torch.from_numpy(np.asarray(ids)).cuda(), out.long()], 1)[:, :-1]
    res, _ = m.prefill(whole.cpu(), never(shape), logits="all")
    logits = res.logits.view(n, -1, shape.vocab)[:, T - 1:]
    got = logits.gather(2, out.long()[..., None])[..., 0]
    tol = 1e-3 if dtype == "f32" else 4e-2
    assert (got >= logits.amax(-1) - tol).all()


def test_drafts_of_the_same_policy_are_kept():
    m = build("f32")
    ids = ai.token_ids(8, SHAPE.vocab, 3, 9)
    out, kept, made, _ = m.generate_drafted(ids, 24, never(), never(), 4)
    assert made and kept >= 0.9 * made
    _, _, plain, _ = m.generate(ids, 24, never())
    # the same greedy tokens, but where two logits are within rounding of each other
    assert (out == plain).float().mean() > 0.9


@pytest.mark.parametrize("temperature", [1.0, 0.7])
def test_sampled_generation_repeats_with_its_generator(temperature):
    m = build("bf16")
    ids = ai.token_ids(9, SHAPE.vocab, 4, 6)
    runs = []
    for seed in (1, 1, 2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        runs.append(m.generate_drafted(ids, 12, never(), early(), 3, temperature, g)[0])
    assert torch.equal(runs[0], runs[1]) and not torch.equal(runs[0], runs[2])


def test_a_verification_pass_is_its_logits_verified():
    m = build("f32")
    n, g, T = 3, 4, 10
    r = torch.Generator().manual_seed(5)
    ids = ai.token_ids(10, SHAPE.vocab, n, T)
    _, cache = m.prefill(ids, never(), s_max=32, logits=None)
    last = torch.randint(0, SHAPE.vocab, (n,), generator=r).int().cuda()
    drafts = torch.randint(0, SHAPE.vocab, (n, g), generator=r).int().cuda()
    q = torch.randn((n, g, SHAPE.vocab), generator=r).cuda()
    u = torch.rand((n, g + 1), generator=r).cuda() * 0.1
    temp = torch.tensor([1.0, 0.0, 0.5], device="cuda")
    pos = torch.full((n,), T, dtype=torch.int32, device="cuda")
    out, kept, res = m.verify(cache, last, drafts, pos, never(), u, q, temp, pos_max=T)
    f = lambda t: t.double().cpu().numpy()
    want = verify(f(res.logits.view(n, g + 1, -1)), f(q), drafts.cpu().numpy(), f(u), None, f(temp))
    assert np.array_equal(out.cpu().numpy(), want[0]) and np.array_equal(kept.cpu().numpy(), want[1])
    # the logits are those of the prompt continued (the same rows in one pass of the prompt)
    whole = torch.cat([torch.from_numpy(np.asarray(ids)), last.cpu().long()[:, None],
                       drafts.cpu().long()], 1)
    ref, _ = m.prefill(whole, never(), logits="all")
    ref = ref.logits.view(n, T + g + 1, -1)[:, T:]
    assert (res.logits.view(n, g + 1, -1) - ref).abs().max() <= 1e-4 * ref.abs().max()
    assert torch.equal(m.draw(res.logits, torch.zeros(n * (g + 1), device="cuda"),
                              torch.zeros(n * (g + 1), device="cuda")), m.greedy(res.logits))


def test_a_verification_pass_exits_token_by_token():
    """Also under the policy by which a prompt's last token decides for all of it: the pass stands
    for decode passes, which do not know that."""
    m = build("f32")
    n, g, T = 3, 5, 10
    ids = ai.token_ids(10, SHAPE.vocab, n, T)
    i32 = dict(dtype=torch.int32, device="cuda")
    drafts = torch.arange(n * g, **i32).view(n, g)
    last, pos = torch.tensor([1, 2, 3], **i32), torch.full((n,), T, **i32)
    u = torch.full((n, g + 1), 0.5, device="cuda")
    out = []
    for prompt_level in (False, True):
        cfg = B.exit_cfg(0.5, SHAPE.n_layers, min_exit_layer=2, prompt_level=prompt_level)
        _, cache = m.prefill(ids, never(), s_max=32, logits=None)
        out.append(m.verify(cache, last, drafts, pos, cfg, u)[2])
        assert cfg.prompt_level == int(prompt_level)
    assert torch.equal(out[0].exit_layer, out[1].exit_layer)
    assert torch.equal(out[0].logits, out[1].logits)


def test_verification_refuses_what_does_not_fit():
    m = build("f32")
    cache = m.new_cache(2, 8)
    z = lambda *d: torch.zeros(d, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="position"):
        m.verify(cache, z(2), z(2, 3), z(2) + 5, never(), torch.zeros((2, 4), device="cuda"))
    with pytest.raises(ValueError, match="sequences"):
        m.verify(cache, z(3), z(3, 3), z(3), never(), torch.zeros((3, 4), device="cuda"))
    with pytest.raises(ValueError, match="drafts"):
        m.generate_drafted(np.zeros((1, 3), np.int64), 4, never(), never(), 0)
    with pytest.raises(ValueError, match="position"):
        m.generate_drafted(np.zeros((1, 3), np.int64), 40, never(), never(), 2, cache=cache)


# ---------------------------------------------------------------- shared pages
def step(m, cache, tok, at):
    n = len(tok)
    i32 = dict(dtype=torch.int32, device="cuda")
    return m.decode_step(cache, torch.tensor(tok, **i32), torch.full((n,), at, **i32), never(),
                         pos_max=at).logits


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("T", [16, 21])
def test_forked_sequences_are_the_prompt_continued(kv, T):
    m = build("bf16")
    prompt = ai.token_ids(11, SHAPE.vocab, 1, T)
    # each sequence for itself
    apart = m.new_paged_cache(3, 12, 8, kv_dtype=kv)
    m.prefill(np.repeat(prompt, 3, 0), never(), logits=None, cache=apart)
    # one sequence, and two forks of it
    shared = m.new_paged_cache(3, 12, 8, kv_dtype=kv)
    shared.reserve({0: T})
    m.prefill(prompt, never(), logits=None, cache=shared)
    shared.fork(0, [1, 2], T)
    full, left = divmod(T, 8)
    assert shared.free_pages == 12 - full - 3 * (left > 0) and shared.shared_pages == full
    for i, tok in enumerate(([1, 2, 3], [4, 5, 6], [9, 8, 7])):
        a, b = step(m, apart, tok, T + i), step(m, shared, tok, T + i)
        # K and V of a prompt may differ by a rounding between a pass over one and over three
        assert (a - b).abs().max() <= 4e-2
    # freed pages come back once the last sequence gives them up
    shared.release(0)
    assert shared.shared_pages == full
    shared.release(2)
    assert shared.shared_pages == 0
    shared.release(1)
    assert shared.free_pages == 12


def test_a_pass_that_writes_over_a_shared_page_copies_it():
    m = build("bf16")
    T = 16
    prompt = ai.token_ids(12, SHAPE.vocab, 1, T)
    c = m.new_paged_cache(2, 8, 8)
    m.prefill(prompt, never(), logits=None, cache=c)
    c.fork(0, 1, T)
    before = step(m, c, [5], T)                            # of sequence 0 alone
    k = c.k.clone()
    old = c.page_table[0, :2].long().tolist()
    # sequence 1 goes back to position 12 and on with other tokens
    i32 = dict(dtype=torch.int32, device="cuda")
    ids = torch.tensor([[5, 30], [5, 31]])
    res, _ = m.prefill(ids, never(), logits="all", cache=c, start=12)
    assert c.page_table[0, 1] != c.page_table[1, 1] and c.page_table[0, 0] == c.page_table[1, 0]
    assert torch.equal(c.k[:, old[0] * 8:old[0] * 8 + 8], k[:, old[0] * 8:old[0] * 8 + 8])
    # both start from the same four tokens of the page
    a, b = (int(c.page_table[j, 1]) * 8 for j in (0, 1))
    assert torch.equal(c.k[:, a:a + 4], c.k[:, b:b + 4])
    assert torch.equal(c.k[0, a + 4], c.k[0, b + 4]) and not torch.equal(c.k[0, a + 5], c.k[0, b + 5])
    assert torch.isfinite(before).all()


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_moved_pages_hold_what_they_held(kv):
    m = build("bf16")
    c = m.new_paged_cache(4, 20, 8, kv_dtype=kv)
    ids = ai.token_ids(13, SHAPE.vocab, 4, 30)
    m.prefill(ids, never(), logits=None, cache=c)
    c.release(0)
    c.truncate(2, 9)
    want = m.prefill(ids[:, :1], never(), logits="all", cache=c, start=9)[0].logits
    used = c.n_pages - c.free_pages
    moved = c.compact()
    assert moved > 0 and int(c.page_table.max()) < used
    got = m.prefill(ids[:, :1], never(), logits="all", cache=c, start=9)[0].logits
    assert torch.equal(got, want)
    c.resize(used + 1)
    assert c.n_pages == used + 1 and c.free_pages == 1 and c.k.shape[1] == (used + 2) * 8
    assert torch.equal(m.prefill(ids[:, :1], never(), logits="all", cache=c, start=9)[0].logits, want)
    c.resize(40)
    assert torch.equal(m.prefill(ids[:, :1], never(), logits="all", cache=c, start=9)[0].logits, want)
    m.prefill(ids, never(), logits=None, cache=c)


def test_generation_over_forks_and_drafts_together():
    """A prompt forked into a batch, and drafted generation from there by its parts."""
    m = build("bf16", quant=True)
    T, n, g = 13, 4, 3
    prompt = ai.token_ids(14, SHAPE.vocab, 1, T)
    c = m.new_paged_cache(n, 30, 8)
    m.prefill(prompt[:, :T - 1], never(), logits=None, cache=c)
    c.fork(0, [1, 2, 3], T - 1)
    gen = torch.Generator(device="cuda").manual_seed(1)
    i32 = dict(dtype=torch.int32, device="cuda")
    last = torch.full((n,), int(prompt[0, T - 1]), **i32)
    pos = torch.full((n,), T - 1, **i32)
    temp = torch.ones(n, device="cuda")
    seqs = [[] for _ in range(n)]
    for _ in range(5):
        tok, drafts, logits = last, [], []
        for k in range(g):
            r = m.decode_step(c, tok, pos + k, early())
            tok = m.draw(r.logits, torch.rand(n, generator=gen, device="cuda"), temp)
            drafts.append(tok)
            logits.append(r.logits)
        out, kept, _ = m.verify(c, last, torch.stack(drafts, 1), pos, never(),
                                torch.rand((n, g + 1), generator=gen, device="cuda"),
                                torch.stack(logits, 1), temp)
        for b in range(n):
            seqs[b] += out[b, :int(kept[b]) + 1].tolist()
        last = out.gather(1, kept.long()[:, None])[:, 0]
        pos = pos + kept + 1
        for b in range(n):
            c.truncate(b, int(pos[b]))
    assert len({tuple(s[:5]) for s in seqs}) > 1
    # what the caches hold is what one pass over each sequence writes
    for b in range(n):
        L = T - 1 + len(seqs[b])
        ids = np.concatenate([prompt[0], seqs[b][:-1]])[None]
        _, ref = m.prefill(ids, never(), logits=None)
        at = c.slots(torch.arange(L, **i32), torch.full((L,), b, **i32)).long()
        err = (c.k[:, at].float() - ref.k[:, :L].float()).abs().max()
        assert err <= 4e-2 * max(1.0, float(ref.k.float().abs().max())), (b, float(err))
