"""adept_paged_attend where scores are minus infinity: keys without weight."""
import pytest
import torch

from tests.test_gpu_paged_attend import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("H,heads,hd", [(4, 2, 64), (2, 2, 128), (2, 1, 32)])
@pytest.mark.parametrize("shape", [[(0, 1, 1), (90, 1, 1), (300, 1, 1)], [(0, 40, 1), (200, 33, 1)]])
def test_keys_whose_score_is_minus_infinity(dt, H, heads, hd, shape):
    """Some of a sequence's keys: as the definition, whether or not a block holds no other.  All of
    another's: zeros, as for an entry that sees no key."""
    print(f"paged attend, scores of -inf, {dt} {H}/{heads}x{hd} {shape}", flush=True)
    c = Case(dt, dt, H, heads, hd, 16, shape, seed=41)
    c.q[..., 0] = c.q[..., 0].abs() + 0.5
    last = c.n_seq - 1
    for t in [*range(0, 150), 170, 199]:
        page = int(c.table[last, t // 16])
        c.pool[0][page * 16 + t % 16, :, 0] = -torch.inf
    at = c.rows.long()
    seq, pos = c.seq[at], c.pos[at]
    if int(pos[seq == last].min()) >= 150:      # keys without weight beside others
        c.check()
    for b in range(c.n_seq):            # now every key of every sequence
        for p in c.table[b][c.table[b] >= 0].tolist():
            c.pool[0][p * 16:(p + 1) * 16, :, 0] = -torch.inf
            c.pool[1][p * 16:(p + 1) * 16].nan_to_num_(0.0)
    assert (c.run() == 0).all()
