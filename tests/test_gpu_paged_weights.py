"""adept_paged_attend of one bf16 token per sequence: the softmax weights keep 16 bits."""
import pytest
import torch

from tests import paged_ref as R
from tests.test_gpu_paged_attend import Case

pytestmark = pytest.mark.gpu

SHAPES = [[(0, 1, 1), (1, 1, 1), (6, 1, 1), (30, 1, 1), (63, 1, 1)], [(127, 1, 1), (300, 1, 1)],
          [(2500, 1, 1)]]


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("H,heads,hd", [(4, 4, 64), (5, 5, 128), (8, 2, 128), (40, 1, 64)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_only_the_result_is_rounded_to_bf16(cache, H, heads, hd, shape):
    """Most results are sums that nearly cancel, so a weight of 8 bits is seen beside them.
    u = 2^-24.  A score's hd products (exact) and sums and a few factors: (hd + 8) u qk, exp2
    2^-22, each of the weight.  A weight as two bf16 values: 2^-16 of it, in the numerator only.
    n keys' sums and rescalings: 2 n u; four waves and up to 126 stretches joined: 2 u each, 260 u.
    The result: 2^-8 of it, and 2^-22 for the quotient."""
    print(f"paged attend, weights, bf16/{cache} {H}/{heads}x{hd} {shape}", flush=True)
    c = Case("bf16", cache, H, heads, hd, 16, shape, seed=31, q_std=0.3)
    out, (ref, wv, qk) = c.run(), c.ref()
    keys = (c.pos[c.rows.long()].double() + 1).view(-1, 1, 1).to(ref.device)
    u = 2.0 ** -24
    d = (hd + 8) * u * qk + 2.0 ** -22 + (2 * keys + 260) * u
    tol = (2 * d + 2.0 ** -16) * wv + (2.0 ** -8 + 2.0 ** -22) * ref.abs() + 1e-30
    worst = ((out.double() - ref).abs() / tol).max().item()
    print(f"  worst error / bound {worst:.3f}", flush=True)
    assert worst <= 1.0


@pytest.mark.parametrize("H,heads,hd", [(4, 4, 64), (8, 2, 128), (2, 1, 32)])
@pytest.mark.parametrize("context", [0, 40, 200, 3000])
def test_infinite_values_that_are_seen(H, heads, hd, context):
    """An infinite V of a seen key: that dim of the result is this infinity, NaN where both signs
    meet, and the other dims are as the definition; nothing of a weight's second part enters."""
    print(f"paged attend, infinite V, {H}/{heads}x{hd} context={context}", flush=True)
    c = Case("bf16", "bf16", H, heads, hd, 16, [(context, 1, 1), (7, 1, 1)], seed=32, q_std=0.3)
    at = [int(c.table[0, t // 16]) * 16 + t % 16 for t in (0, context // 3, context // 2, context)]
    for d, signs in enumerate([(1, 1, 1, 1), (-1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 0, -1), (0, -1, -1, 1)]):
        for slot, sign in zip(at, signs):
            if sign:
                c.pool[1][slot, :, 3 * d] = sign * torch.inf
    out, (ref, wv, qk) = c.run().double(), c.ref()
    assert torch.equal(out.isnan(), ref.isnan())
    assert torch.equal(out.isposinf(), ref.isposinf()) and torch.equal(out.isneginf(), ref.isneginf())
    assert out[0].isposinf().any() and not out[1].isinf().any()
    fine = torch.isfinite(ref)
    tol = R.bound(c.dt, ref, wv, qk)
    assert ((out - ref).abs() <= tol)[fine].all()
