"""Every form of the 4-bit product with every epilogue (the sizes of quant_forms.py): layers against
the oracle, plain products against sums in 64 bits."""
import math

import pytest
import torch

from paper_2601_03700_amd import binding as B
from tests import quant_forms as Q
from tests.test_gpu_quant import check, pack, rand, unpack
from tests.test_gpu_quant_layers import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,rows", Q.LAYERS, ids=[
    f"{s.family}-{s.d_model}-{s.n_heads}x{s.head_dim}-{s.d_ff}-{r}" for s, r in Q.LAYERS])
def test_layers(shape, rows):
    run(shape, rows, 1)


@pytest.mark.parametrize("m,n,k", Q.PRODUCTS)
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_products(m, n, k, out):
    qw = pack(rand(n, n, k) * 0.05)
    wide = rand(m + k, m, k + 8).to(torch.bfloat16).cuda()
    x, bias = wide[:, :k], rand(3, n).to(torch.bfloat16).cuda()
    y = torch.full((m, n + 3), math.nan, dtype=out, device="cuda")
    B.quant_linear(x, qw, y[:, 1:1 + n], bias=bias)
    check(y[:, 1:1 + n], x, unpack(qw), bias)
    assert y[:, 0].isnan().all() and y[:, 1 + n:].isnan().all()
