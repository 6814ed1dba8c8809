"""adept_paged_attend over eight and more K/V heads, whose work is dealt to the chip's eight parts in
runs: several tiles a head, cut keys, counts that eight does not divide."""
import pytest
import torch

from tests.test_gpu_paged_attend import TYPES, Case

pytestmark = pytest.mark.gpu

SHAPES = {"a prompt": [(0, 257, 1)], "cut keys": [(700, 9, 1)], "several": [(900, 70, 0.8), (0, 33, 1), (5, 140, 1)]}


@pytest.mark.parametrize("dt,cache", TYPES)
@pytest.mark.parametrize("H,heads,hd", [(8, 8, 64), (11, 11, 64), (25, 25, 64), (36, 9, 128), (16, 16, 128)])
@pytest.mark.parametrize("shape", SHAPES)
def test_matches_definition(dt, cache, H, heads, hd, shape):
    print(f"paged attend, {H}/{heads}x{hd} {dt}/{cache} {shape}", flush=True)
    Case(dt, cache, H, heads, hd, 16, SHAPES[shape], seed=13).check()


@pytest.mark.parametrize("dt,cache", TYPES)
def test_scattered_sequences(dt, cache):
    """Two sequences' entries in turn: more tiles than the host counts on, none of them cut."""
    print(f"paged attend, entries in turn, {dt}/{cache}", flush=True)
    c = Case(dt, cache, 9, 9, 64, 16, [(300, 60, 1), (20, 60, 1)], seed=14)
    turn = torch.stack([torch.arange(60), torch.arange(60, 120)], 1).view(-1)
    c.rows, c.q = c.rows[turn], c.q[turn]
    c.check()
