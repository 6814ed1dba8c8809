"""binding.layer_step_paged asks for the cache of all layers, on the host."""
import pytest
import torch

from paper_2601_03700_amd import binding as B
from paper_2601_03700_amd.model import PagedKVCache


def step(kv, n_layers):
    a = B.LayerArgs()
    a.n_layers, a.n_seq, a.n_tok = n_layers, 3, 5
    B.layer_step_paged(a, kv, torch.zeros((3, 4), dtype=torch.int32), 1,
                       torch.zeros(5, dtype=torch.int32))


@pytest.mark.parametrize("kind", ["bf16", "f32", "fp8"])
def test_a_descriptor_with_fewer_layers_behind_it(kind):
    """The kernels would write behind the cache."""
    c = PagedKVCache(3, 2, 16, 3, 6, 4, 4, kind, "cpu")
    for kv, n in ((c.kv, 4), (c.layer_kv(2), 3), (c.layer_kv(3), 2)):
        with pytest.raises(B.AdeptError, match="layers"):
            step(kv, n)
    for kv, n in ((c.kv, 3), (c.layer_kv(2), 2), (c.layer_kv(3), 1)):
        with pytest.raises(B.AdeptError, match="current HIP device"):    # passes that check
            step(kv, n)


def test_scales_of_fewer_layers():
    k, v = (torch.zeros((3, 8, 2, 64), dtype=torch.uint8) for _ in range(2))
    ks, vs = torch.zeros((3, 8, 2), dtype=torch.uint8), torch.zeros((2, 8, 2), dtype=torch.uint8)
    with pytest.raises(B.AdeptError, match="layers"):
        step(B.paged_kv(k[0], v[0], 4, ks[0], vs[0]), 3)
