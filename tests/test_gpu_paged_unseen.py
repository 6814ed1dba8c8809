"""adept_paged_attend over 8-bit caches whose unseen slots hold anything, scale bytes included."""
import math

import pytest
import torch

import adept_inputs as ai
from paper_2601_03700_amd import binding as B
from tests.test_gpu_paged_attend import Case
from tests.test_gpu_paged_model import LLAMA, Checker, build

pytestmark = pytest.mark.gpu


def unwritten(c, byte):
    """Slots that no entry may read get NaN codes and the scale byte `byte`, slot 0 among them: page
    0 changes places with a page that no table names."""
    used = set(c.table[c.table >= 0].tolist())
    page = c.page
    spare = next(p for p in range(c.pool[0].shape[0] // page) if p and p not in used)
    if 0 in used:
        for x in (*c.pool, *c.scales):
            x[spare * page:(spare + 1) * page] = x[:page]
        c.table[c.table == 0] = spare
    seen = torch.zeros(c.pool[0].shape[0], dtype=torch.bool)
    for b in range(c.n_seq):
        n = 1 + max([int(p) for p, s in zip(c.pos, c.seq) if s == b], default=-1)
        t = torch.arange(n)
        seen[c.table[b].long()[t // page] * page + t % page] = True
    assert not seen[0]
    for p, s in zip(c.pool, c.scales):
        p[~seen], s[~seen] = 0x7f, byte
    return seen


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("H,heads,hd", [(4, 4, 64), (8, 2, 128), (40, 1, 128), (2, 1, 256)])
@pytest.mark.parametrize("shape", [[(0, 1, 1), (62, 1, 1), (127, 1, 1), (300, 1, 1)],
                                   [(0, 40, 1), (60, 70, 0.8), (5, 3, 1)]])
@pytest.mark.parametrize("byte", [255, 0])
def test_scales_of_slots_never_written(dt, H, heads, hd, shape, byte):
    """255 is no scale (its exponent bits are those of infinity and NaN); what is not seen has no
    influence, whatever it holds: ends of sequences, dead slots and pages that are not there."""
    print(f"paged attend, unseen scales {byte}, {dt} {H}/{heads}x{hd} {shape}", flush=True)
    c = Case(dt, "fp8", H, heads, hd, 16, shape, seed=5)
    seen = unwritten(c, byte)
    out = c.check()
    assert torch.isfinite(out).all()
    g = torch.Generator().manual_seed(1)
    c.live = (torch.rand(seen.shape, generator=g) < 0.8).to(torch.uint8)
    for p, s in zip(c.pool, c.scales):
        p[c.live == 0], s[c.live == 0] = 0x7f, byte
    c.table[1, 1] = -1
    assert torch.isfinite(c.check()).all()


@pytest.mark.parametrize("chunk", [1, 33])
def test_scales_of_slots_never_written_leave_the_bits(chunk):
    """The same result, to the bit, whatever the unseen slots hold."""
    print(f"paged attend, unseen scales, bits, chunk={chunk}", flush=True)
    c = Case("bf16", "fp8", 8, 2, 128, 16, [(700, chunk, 1), (70, chunk, 1)], seed=2)
    unwritten(c, 120)
    want = c.check().clone()
    for byte in (255, 0, 127):
        unwritten(c, byte)
        assert torch.equal(c.run(), want)


@pytest.mark.parametrize("fused", [True, False])
def test_decode_over_a_cache_whose_first_page_is_another_sequences(fused):
    """Page 0 is reserved for a sequence that no pass has run yet: its scales hold anything."""
    print(f"paged model, first page unwritten, fused={fused}", flush=True)
    shape, T = LLAMA, 21
    model = build(shape, "bf16", kv_fused=fused)
    cfg = B.exit_cfg(math.inf, shape.n_layers)
    cache = model.new_paged_cache(2, n_pages=8, page_size=8, kv_dtype="fp8")
    for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        t.fill_(0x7f if t.dim() == 4 else 255)
    cache.reserve({1: 8})
    assert int(cache.page_table[1, 0]) == 0
    check = Checker(model, cache)
    ids = ai.token_ids(4, shape.vocab, 1, T)
    res, _ = model.prefill(ids, cfg, cache=cache, logits="last", on_layer=check)
    nxt = model.greedy(res.logits)
    for j in range(3):
        pos = torch.full((1,), T + j, dtype=torch.int32, device="cuda")
        res = model.decode_step(cache, nxt, pos, cfg, on_layer=check)
        assert torch.isfinite(res.logits).all()
        nxt = model.greedy(res.logits)
    assert check.layers == 4 * shape.n_layers
