"""adept_paged_attend of f32 queries, held to the rounding of f32 at the lengths in question."""
import pytest
import torch

from tests import paged_ref as R
from tests.test_gpu_paged_attend import Case

# scores near zero, so that the weights and the sums are what rounds
Q_STD = 0.05
SHAPES = [[(0, 1, 1), (1, 1, 1), (6, 1, 1), (30, 1, 1)], [(0, 8, 1), (2, 5, 1)],
          [(0, 64, 1)], [(40, 24, 1), (0, 33, 0.8)]]
HEADS = [(4, 4, 64), (8, 2, 128), (3, 3, 32), (2, 1, 256), (2, 2, 16)]


def bound(hd, capacity, keys, ref, wv, qk):
    """u = 2^-24.  A score is off by at most hd products and sums and a few factors, (hd + 8) u qk,
    and so is its weight, relative to it; exp2 by 2^-22.  The numerator of n keys: each is added
    once and what was there is scaled at most once, 2 n u of wv; the normaliser the same; parts of
    64 keys of the table's capacity, up to 32, are joined with two roundings each.  The quotient:
    a reciprocal and a product, 2^-22 of the result."""
    u = 2.0 ** -24
    joins = min(32, -(-capacity // 64))
    d = (hd + 8) * u * qk + 2.0 ** -22 + (2 * keys + 2 * joins + 4) * u
    return 2 * d * wv + 2.0 ** -22 * ref.abs() + 1e-30


def case(cache, H, heads, hd, shape):
    return Case("f32", cache, H, heads, hd, 16, shape, seed=21, q_std=Q_STD)


def keys_of(c):
    return (c.pos[c.rows.long()].double() + 1).view(-1, 1, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("cache", ["f32", "fp8"])
@pytest.mark.parametrize("H,heads,hd", HEADS)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_f32_rounding(cache, H, heads, hd, shape):
    print(f"paged attend, f32 rounding, f32/{cache} {H}/{heads}x{hd} {shape}", flush=True)
    c = case(cache, H, heads, hd, shape)
    out, (ref, wv, qk) = c.run(), c.ref()
    tol = bound(hd, c.table.shape[1] * c.page, keys_of(c).to(ref.device), ref, wv, qk)
    worst = ((out.double() - ref).abs() / tol).max().item()
    print(f"  worst error / bound {worst:.3f}", flush=True)
    assert worst <= 1.0


@pytest.mark.parametrize("bits", [11, 13])
@pytest.mark.parametrize("shape", SHAPES[:2], ids=str)
def test_the_bound_sees_weights_of_fewer_bits(bits, shape):
    """The definition itself with the softmax weights rounded to 11 or 13 bits is beyond it."""
    c = case("f32", 4, 4, 64, shape)
    at, k, v = c.rows.long(), c.pool[0].double(), c.pool[1].double()
    ref, wv, qk = R.attend(c.q, k, v, c.table, c.page, c.pos[at], c.seq[at], c.scale)
    off = ref.clone()
    for i, r in enumerate(at.tolist()):
        t = torch.arange(int(c.pos[r]) + 1)
        slot = c.table[c.seq[r]].long()[t // c.page] * c.page + t % c.page
        for h in range(4):
            s = k[slot, h] @ c.q[i, h].double() * c.scale
            m, e = torch.frexp(torch.exp(s - s.max()))
            off[i, h] = torch.ldexp(torch.round(m * 2 ** bits) / 2 ** bits, e) @ v[slot, h] \
                / torch.exp(s - s.max()).sum()
    tol = bound(64, c.table.shape[1] * c.page, keys_of(c), ref, wv, qk)
    assert ((off - ref).abs() / tol).max() > 1.0
