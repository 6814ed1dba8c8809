"""adept_verify_drafts against its definition in 64 bits.  Tokens and counts are equal: the library
computes in 64 bits too, and a border within its rounding of a random number (about 1e-14 of a
token's probability) is not met by these inputs."""
import math

import numpy as np
import pytest
import torch

from paper_2601_03700_amd import binding as B
from tests.verify_ref import verify

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def inputs(seed, n, g, V, dtype, agree=0.7):
    r = torch.Generator().manual_seed(seed)
    target = torch.randn((n, g + 1, V), generator=r) * 2
    draft = target[:, :g] + agree * torch.randn((n, g, V), generator=r)
    target, draft = target.to(DT[dtype]), draft.to(DT[dtype])
    law = torch.softmax(draft.float(), -1)
    tokens = torch.multinomial(law.reshape(-1, V), 1, generator=r).view(n, g) if g else \
        torch.zeros((n, 0), dtype=torch.long)
    u = torch.rand((n, g + 1), generator=r)
    return target, draft, tokens.to(torch.int32), u


def run(target, draft, tokens, u, n_draft=None, temperature=None, views=None):
    up = lambda t: None if t is None else t.cuda()
    n, rows, V = target.shape
    t, d = (up(target), up(draft)) if views is None else views
    out = torch.full((n, rows), -7, dtype=torch.int32, device="cuda")
    kept = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    ws = torch.full((B.verify_drafts_workspace_bytes(n, rows - 1, V),), 0xff, dtype=torch.uint8,
                    device="cuda")
    B.verify_drafts(t, d, up(tokens), up(u), out, kept, up(n_draft), up(temperature), ws)
    return out.cpu().numpy(), kept.cpu().numpy()


def want(target, draft, tokens, u, n_draft=None, temperature=None):
    f = lambda t: None if t is None else t.double().numpy()
    return verify(f(target), f(draft), tokens.numpy(), u.double().numpy(),
                  None if n_draft is None else n_draft.numpy(), f(temperature))


def same(a, b):
    assert np.array_equal(a[1], b[1])
    assert np.array_equal(a[0], b[0])


SHAPES = [(1, 0, 1), (1, 1, 1), (2, 1, 7), (3, 4, 1000), (5, 3, 2047), (4, 2, 2048), (4, 2, 2049),
          (6, 5, 4099), (2, 16, 50257), (130, 2, 513), (3, 70, 300)]


@pytest.mark.parametrize("n,g,V", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["drafter", "lookup", "greedy"])
def test_against_the_definition(n, g, V, dtype, kind):
    target, draft, tokens, u = inputs(n * 100 + g + V, n, g, V, dtype)
    temp = None
    if kind == "greedy":
        temp = torch.zeros(n)
        # half of the drafts are what the model would say
        best = target[:, :g].float().argmax(-1).to(torch.int32)
        tokens = torch.where(torch.arange(n)[:, None] % 2 == 0, best, tokens)
    draft = None if kind == "lookup" else draft
    same(run(target, draft, tokens, u, temperature=temp), want(target, draft, tokens, u, None, temp))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_counts_and_temperatures_of_each_sequence(dtype):
    n, g, V = 24, 6, 3001
    target, draft, tokens, u = inputs(5, n, g, V, dtype)
    count = torch.tensor([k % 9 - 1 for k in range(n)], dtype=torch.int32)     # -1 .. 7
    temp = torch.tensor([1.0, 0.0, 0.5, 2.0, -1.0, math.nan, 0.01, math.inf] * 3)
    same(run(target, draft, tokens, u, count, temp), want(target, draft, tokens, u, count, temp))
    same(run(target, None, tokens, u, count, temp), want(target, None, tokens, u, count, temp))


def test_rows_behind_the_drafts_are_not_used():
    n, g, V = 5, 4, 777
    target, draft, tokens, u = inputs(6, n, g, V, "f32")
    count = torch.tensor([0, 1, 2, 3, 4], dtype=torch.int32)
    ref = run(target, draft, tokens, u, count)
    for b in range(n):
        target[b, b + 1:] = math.inf
        draft[b, b:] = math.nan
        tokens[b, b:] = -5
    same(run(target, draft, tokens, u, count), ref)


def test_masked_infinite_and_missing_logits():
    n, g, V = 10, 2, 600
    target, draft, tokens, u = inputs(7, n, g, V, "f32")
    ninf = -math.inf
    target[0, 0, ::2] = ninf                          # a mask; the draft may lie in it
    target[1, 0] = ninf                               # no row at all
    target[2, :] = ninf
    target[3, 0, 5], target[3, 0, 77] = math.inf, math.inf
    target[4, 1, 100:] = math.nan
    draft[5, 0] = ninf                                # the drafter's row says nothing
    draft[6, 0, 9] = math.inf
    target[7, 0] = torch.finfo(torch.float32).min     # the type's lowest value everywhere
    tokens[8, 0], tokens[9, 1] = V, -1
    target[9, 2] = math.nan
    same(run(target, draft, tokens, u), want(target, draft, tokens, u))
    same(run(target, None, tokens, u), want(target, None, tokens, u))
    zero = torch.zeros(n)
    same(run(target, draft, tokens, u, None, zero), want(target, draft, tokens, u, None, zero))


@pytest.mark.parametrize("last", [0.0, 0.99999994, 1.0])
def test_the_ends_of_the_random_numbers(last):
    n, g, V = 6, 2, 5000
    target, draft, tokens, u = inputs(8, n, g, V, "f32")
    target[:, :, :40] = -math.inf
    target[:, :, 4900:] = -math.inf
    u[:, g] = last
    u[3:, 0] = 1.0                                    # never below p / q = 1
    draft[4:] = target[4:, :g]                        # p - q leaves nothing
    out, kept = run(target, draft, tokens, u)
    same((out, kept), want(target, draft, tokens, u))
    assert ((out >= 40) & (out < 4900) | (out == -1)).all()


def test_ties_go_to_the_lowest_token():
    n, g, V = 3, 2, 5003
    target = torch.zeros((n, g + 1, V), dtype=torch.bfloat16)
    target[1, :, 4100:] = 3
    target[2, :, [17, 2100, 5002]] = 5
    tokens = torch.tensor([[0, 0], [4100, 4101], [17, 2100]], dtype=torch.int32)
    out, kept = run(target, None, tokens, torch.zeros(n, g + 1), None, torch.zeros(n))
    assert kept.tolist() == [2, 1, 1]
    assert out.tolist() == [[0, 0, 0], [4100, 4100, -1], [17, 17, -1]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_any_stride_and_alignment(dtype):
    n, g, V = 4, 3, 1237
    target, draft, tokens, u = inputs(9, n, g, V, dtype)
    ref = want(target, draft, tokens, u)
    for pad, off in ((0, 1), (3, 0), (11, 5)):
        views = []
        for x in (target, draft):
            wide = torch.full((n, x.shape[1], V + pad + off), math.nan, dtype=DT[dtype], device="cuda")
            wide[:, :, off:off + V] = x.cuda()
            views.append(wide[:, :, off:off + V])
        same(run(target, draft, tokens, u, views=views), ref)


def test_every_token_is_distributed_as_the_model():
    """The first emitted token over 40000 sequences: drafts from q, frequencies as p.  Of each token
    within five deviations of a binomial."""
    n, V = 40000, 6
    r = torch.Generator().manual_seed(3)
    p = torch.tensor([0.05, 0.4, 0.1, 0.25, 0.15, 0.05])
    q = torch.tensor([0.3, 0.1, 0.1, 0.2, 0.05, 0.25])
    tokens = torch.multinomial(q, n, True, generator=r).to(torch.int32)[:, None]
    u = torch.rand((n, 2), generator=r)
    target = p.log().expand(n, 2, V).contiguous()
    out, kept = run(target, q.log().expand(n, 1, V).contiguous(), tokens, u)
    got = np.bincount(out[:, 0], minlength=V) / n
    assert (abs(got - p.numpy()) < 5 * np.sqrt(p.numpy() * (1 - p.numpy()) / n)).all(), got
    out, _ = run(target, None, tokens, u)
    got = np.bincount(out[:, 0], minlength=V) / n
    assert (abs(got - p.numpy()) < 5 * np.sqrt(p.numpy() * (1 - p.numpy()) / n)).all(), got
    assert 0.5 < kept.mean() < 0.75        # sum of min(p, q) = 0.6


def test_captured_and_replayed_beside_eager_work():
    n, g, V = 8, 4, 32000
    a, b = inputs(11, n, g, V, "f32"), inputs(12, n, g, V, "f32")
    dev = [x.cuda() for x in a]
    out = torch.empty((n, g + 1), dtype=torch.int32, device="cuda")
    kept = torch.empty(n, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.verify_drafts_workspace_bytes(n, g, V), dtype=torch.uint8, device="cuda")
    call = lambda: B.verify_drafts(*dev, out, kept, workspace=ws)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        x = (a, b)[i % 2]
        for d, s in zip(dev, x):
            d.copy_(s)
        out.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        got = out.cpu().numpy(), kept.cpu().numpy()
        same(got, want(*x))
        same(run(*x), got)


def test_two_calls_at_once():
    n, g, V = 16, 5, 32000
    a, b = inputs(13, n, g, V, "f32"), inputs(14, n, g, V, "bf16")
    calls = []
    for x in (a, b):
        dev = [t.cuda() for t in x]
        calls.append((dev, torch.empty((n, g + 1), dtype=torch.int32, device="cuda"),
                      torch.empty(n, dtype=torch.int32, device="cuda"),
                      torch.empty(B.verify_drafts_workspace_bytes(n, g, V), dtype=torch.uint8,
                                  device="cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(3):
        for dev, out, kept, ws, s in calls:
            B.verify_drafts(*dev, out, kept, workspace=ws, stream=s)
    torch.cuda.synchronize()
    for x, (_, out, kept, _, _) in zip((a, b), calls):
        same((out.cpu().numpy(), kept.cpu().numpy()), want(*x))
