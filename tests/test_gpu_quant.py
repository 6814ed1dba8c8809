"""Weights in 4 bits: packed, read back, and multiplied with few rows."""
import math

import numpy as np
import pytest
import torch

from paper_2601_03700_amd import binding as B
from tests.quant_ref import quantised

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def pack(w, mats=1, mat=0):
    qw = B.quant_weights(*w.shape, "cuda", mats)
    qw.codes.fill_(0x77)
    qw.scales.fill_(0x77)
    B.quant_pack(w.cuda(), qw, mat)
    return qw


def unpack(qw, dtype=torch.float32, mat=0):
    out = torch.full((qw.n, qw.k), math.nan, dtype=dtype, device="cuda")
    B.quant_unpack(qw, out, mat)
    return out


@pytest.mark.parametrize("n,k", [(1, 1), (1, 8), (3, 31), (16, 32), (17, 33), (5, 128), (40, 136),
                                 (33, 257), (64, 96)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_are_the_definition(n, k, dtype):
    w = (rand(n + k, n, k) * torch.logspace(-6, 4, n)[:, None]).to(DT[dtype])
    want = torch.from_numpy(quantised(w.double().numpy()))
    qw = pack(w)
    for back in (torch.float32, torch.bfloat16):       # exact in both
        assert torch.equal(unpack(qw, back).double().cpu(), want)
    # what has the values keeps them
    again = pack(want.float())
    assert torch.equal(unpack(again).double().cpu(), want)


def test_ties_borders_and_extremes():
    ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5]
    rows = [[7.0] + ties + [-t for t in ties],
            [np.nextafter(np.float32(7), np.float32(8))] + ties,   # the next power of two
            [7.0] + [float(np.nextafter(np.float32(t), np.float32(9))) for t in ties],
            [7.0] + [float(np.nextafter(np.float32(t), np.float32(0))) for t in ties],
            [3e38, 1.0], [1e-38, 1e-45, -2e-39], [2.0 ** -100, 2.0 ** -102], [0.0, -0.0],
            [-6.0, 1e-20], [448.0, 1.0]]
    w = torch.zeros((len(rows), 32))
    for i, r in enumerate(rows):
        w[i, :len(r)] = torch.tensor(r, dtype=torch.float32)
    want = torch.from_numpy(quantised(w.double().numpy()))
    assert torch.equal(unpack(pack(w)).double().cpu(), want)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_group_that_is_not_finite_is_nan(bad):
    w = rand(1, 20, 100)
    w[3, 40] = bad
    qw = pack(w)
    got = unpack(qw).cpu()
    assert got[3, 32:64].isnan().all() and got.isnan().sum() == 32
    y = torch.empty((2, 20), device="cuda")
    B.quant_linear(torch.zeros((2, 104), dtype=torch.bfloat16, device="cuda"),
                   pack(torch.nn.functional.pad(w, (0, 4))), y)
    assert y[:, 3].isnan().all() and y.isnan().sum() == 2      # 0 times NaN


def test_views_stacks_and_what_is_behind():
    w = rand(2, 30, 77)
    wide = torch.full((30, 90), math.nan)
    wide[:, 5:82] = w
    for dt in (torch.float32, torch.bfloat16):
        src = wide.to(dt).cuda()[:, 5:82]
        qw = B.quant_weights(30, 77, "cuda", 3)
        before = qw.codes.fill_(0x11).clone()
        B.quant_pack(src, qw, 1)
        assert torch.equal(qw.codes[0], before[0]) and torch.equal(qw.codes[2], before[2])
        back = torch.full((30, 90), 5.0, dtype=dt, device="cuda")
        B.quant_unpack(qw, back[:, 3:80], 1)
        want = torch.from_numpy(quantised(w.to(dt).double().numpy()))
        assert torch.equal(back[:, 3:80].double().cpu(), want)
        assert (back[:, :3] == 5).all() and (back[:, 80:] == 5).all()


# Products of bf16 numbers are exact in f32; a sum of k of them in f32, in any order and rounded or
# cut at each step, is off by at most k 2^-23 times the sum of the magnitudes (and rounding the
# result: bf16 2^-8 of it).
def check(y, x, w, bias=None):
    x, w = x.double().cpu(), w.double().cpu()
    ref, mag = x @ w.T, x.abs() @ w.abs().T
    if bias is not None:
        ref, mag = ref + bias.double().cpu(), mag + bias.double().abs().cpu()
    tol = (x.shape[1] + 2) * 2.0 ** -23 * mag
    if y.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * ref.abs() + 2.0 ** -8 * tol
    else:
        tol = tol + 2.0 ** -24 * ref.abs()
    err = (y.double().cpu() - ref).abs()
    assert (err <= tol).all(), float((err / tol.clamp(min=1e-300)).max())


CASES = [(1, 1, 8), (1, 16, 128), (2, 17, 40), (3, 33, 136), (5, 5, 1000), (16, 48, 256),
         (17, 100, 264), (24, 1600, 1600), (32, 31, 512), (33, 130, 776), (64, 64, 1160),
         (64, 8200, 96), (65, 50, 128), (130, 40, 392), (1, 12288, 512), (7, 1000, 4096),
         (20, 8199, 128), (16, 512, 11008)]


@pytest.mark.parametrize("m,n,k", CASES)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_products(m, n, k, out):
    qw = pack(rand(n, n, k) * 0.05)
    x = rand(m + k, m, k).to(torch.bfloat16).cuda()
    y = torch.full((m, n), math.nan, dtype=DT[out], device="cuda")
    B.quant_linear(x, qw, y)
    check(y, x, unpack(qw))
    bias = rand(3, n).to(torch.bfloat16).cuda()
    y.fill_(math.nan)
    B.quant_linear(x, qw, y, bias=bias)
    check(y, x, unpack(qw), bias)


@pytest.mark.parametrize("m", [1, 5, 20, 40, 100])
def test_row_lists_counts_strides_and_what_is_behind(m):
    n, k = 77, 200
    qw = pack(rand(4, n, k))
    wide = rand(5, 120, k + 56).to(torch.bfloat16).cuda()
    x = wide[:, 16:16 + k]
    rows = torch.randperm(120, generator=torch.Generator().manual_seed(m))[:m].to(torch.int32).cuda()
    for live in (0, 1, m // 2, m, m + 9):
        count = torch.tensor([live], dtype=torch.int32, device="cuda")
        for dt in (torch.float32, torch.bfloat16):
            y = torch.full((m + 2, n + 9), 3.0, dtype=dt, device="cuda")
            B.quant_linear(x, qw, y[:, 5:5 + n], rows=rows, n_rows=count)
            c = min(live, m)
            check(y[:c, 5:5 + n], x[rows.long()[:c]], unpack(qw))
            assert (y[c:] == 3).all() and (y[:, :5] == 3).all() and (y[:, 5 + n:] == 3).all()


def test_rows_and_k_that_are_not_there_have_no_influence():
    """NaN behind k (in the row's padding) and in rows that the list leaves out."""
    n, k = 48, 72
    qw = pack(rand(6, n, k))
    wide = torch.full((9, 128), math.nan, dtype=torch.bfloat16, device="cuda")
    wide[:, :k] = rand(7, 9, k).cuda()
    wide[0] = math.nan
    rows = torch.tensor([3, 8, 3], dtype=torch.int32, device="cuda")
    y = torch.empty((3, n), device="cuda")
    B.quant_linear(wide[:, :k], qw, y, rows=rows)
    check(y, wide[rows.long(), :k], unpack(qw))
    # a row of infinities stays by itself
    x = rand(8, 4, k).to(torch.bfloat16).cuda()
    x[2, 5] = math.inf
    y = torch.empty((4, n), device="cuda")
    B.quant_linear(x, qw, y)
    keep = [0, 1, 3]
    check(y[keep], x[keep], unpack(qw))
    assert not y[2].isfinite().any()


def test_captured_and_replayed():
    n, k, m = 4096, 1024, 9
    qw = pack(rand(9, n, k))
    x = torch.empty((m, k), dtype=torch.bfloat16, device="cuda")
    y = torch.empty((m, n), device="cuda")
    x.copy_(rand(10, m, k))
    B.quant_linear(x, qw, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.quant_linear(x, qw, y)
    for i in range(3):
        x.copy_(rand(20 + i, m, k))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check(y, x, unpack(qw))
        eager = torch.empty_like(y)
        B.quant_linear(x, qw, eager)
        assert torch.equal(eager, y)
