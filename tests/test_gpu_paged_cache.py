"""adept_paged_store and adept_paged_load against the definition in 64 bits: codes and values to
the bit."""
import math

import pytest
import torch

from paper_2601_03700_amd import binding as B
from tests import paged_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rows_of(n, heads, hd, dtype, seed):
    """Rows of many sizes; some with zeros, the smallest and largest values, infinities, NaN."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, heads, hd), generator=g) * torch.pow(
        2.0, torch.randint(-40, 40, (n, heads, 1), generator=g).float())
    flat = x.view(-1, hd)
    m = flat.shape[0]
    big = 3.38e38 if dtype == torch.bfloat16 else 3.4e38
    special = [(0, 0.0), (1, 1e-42), (2, 1e-36), (3, big)]
    for r, val in special:
        if r < m:
            flat[r] = val * torch.sign(flat[r])
    if m > 8:
        flat[4, 3], flat[5, 1], flat[5, hd - 1] = math.inf, -math.inf, math.nan
        flat[6], flat[7] = math.nan, math.inf
        flat[8, 0] = 448.0 * 2.0 ** 30          # on the line between two scales
        flat[8, 1:] = 5.0
    if m > 20:          # every halfway point between codes, the largest value fixing E = 0
        mags = R.e4m3_values()[:127]
        mid = ((mags[1:] + mags[:-1]) / 2).float()
        for r in range(9, 20):
            pick = torch.randint(0, mid.numel(), (hd,), generator=g)
            flat[r] = mid[pick] * torch.sign(torch.randn(hd, generator=g))
            flat[r, 0] = 400.0
    return x.to(dtype)


CASES = [("bf16", 3, 128, 16, 50), ("bf16", 1, 16, 1, 33), ("bf16", 25, 64, 8, 7),
         ("bf16", 2, 256, 1024, 9), ("f32", 2, 128, 32, 50), ("f32", 5, 32, 4, 40),
         ("f32", 3, 256, 2, 12), ("bf16", 40, 128, 16, 1), ("f32", 1, 64, 64, 200)]


@pytest.mark.parametrize("dt,heads,hd,page,n", CASES)
def test_quantise_and_read_back(dt, heads, hd, page, n):
    print(f"paged round trip {dt} heads={heads} hd={hd} page={page} n={n}", flush=True)
    dtype = R.TDT[dt]
    k, v = rows_of(n, heads, hd, dtype, 1), rows_of(n, heads, hd, dtype, 2)
    slots = -(-(n + 5) // page) * page
    g = torch.Generator().manual_seed(n)
    slot = torch.randperm(slots, generator=g)[:n].to(torch.int32)
    pool = [torch.full((slots, heads, hd), 0x55, dtype=torch.uint8, device=DEV) for _ in range(2)]
    sc = [torch.full((slots, heads), 9, dtype=torch.uint8, device=DEV) for _ in range(2)]
    kv = B.paged_kv(pool[0], pool[1], page, sc[0], sc[1])
    B.paged_store(kv, k.to(DEV), v.to(DEV), slot.to(DEV))
    others = torch.ones(slots, dtype=torch.bool)
    others[slot.long()] = False
    for x, p, s in ((k, pool[0].cpu(), sc[0].cpu()), (v, pool[1].cpu(), sc[1].cpu())):
        val, E = R.quantised(x)
        assert torch.equal(s[slot.long()].long() - 127, E)
        got = R.e4m3_values()[p[slot.long()].long()]
        assert torch.equal(got.isnan(), val.isnan())
        assert torch.equal(got.nan_to_num(), val.nan_to_num())
        assert (p[others] == 0x55).all() and (s[others] == 9).all()
    # read back, exactly, in both types
    for out_t in (torch.float32, torch.bfloat16):
        ko, vo = (torch.empty((n, heads, hd), dtype=out_t, device=DEV) for _ in range(2))
        B.paged_load(kv, slot.to(DEV), ko, vo)
        for o, p, s in ((ko, pool[0], sc[0]), (vo, pool[1], sc[1])):
            want = R.cache_values(p.cpu()[slot.long()], s.cpu()[slot.long()])
            got = o.double().cpu()
            assert torch.equal(got.isnan(), want.isnan())
            assert torch.equal(got.nan_to_num(), want.nan_to_num())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_every_code_at_every_scale(dt):
    print(f"paged load, every code and scale, {dt}", flush=True)
    E = torch.arange(27, 228, dtype=torch.uint8)
    codes = torch.arange(256, dtype=torch.uint8).view(1, 1, 256).repeat(E.numel(), 1, 1)
    dev = codes.to(DEV)
    kv = B.paged_kv(dev, dev.flip(2).contiguous(), 1, E.view(-1, 1).to(DEV), E.view(-1, 1).to(DEV))
    n = E.numel()
    k, v = (torch.empty((n, 1, 256), dtype=R.TDT[dt], device=DEV) for _ in range(2))
    B.paged_load(kv, torch.arange(n, dtype=torch.int32, device=DEV), k, v)
    want = R.cache_values(codes, E.view(-1, 1))
    for got in (k, v.flip(2)):
        got = got.double().cpu()
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(got.nan_to_num(), want.nan_to_num())


@pytest.mark.parametrize("dt,heads,hd", [("bf16", 3, 64), ("f32", 2, 128), ("bf16", 32, 128),
                                         ("f32", 7, 16)])
@pytest.mark.parametrize("fp8", [False, True])
def test_lists_strides_and_missing_slots(dt, heads, hd, fp8):
    """Rows out of a wider projection, a list of some of them with a count on the device below its
    length, slots outside the cache; what is not written stays."""
    print(f"paged store, lists and strides {dt} {heads}x{hd} fp8={fp8}", flush=True)
    dtype, n, page, slots = R.TDT[dt], 37, 16, 96
    g = torch.Generator().manual_seed(5)
    wide = torch.randn((n, 3 * heads * hd + 8), generator=g).to(dtype).to(DEV)
    k = wide[:, heads * hd:2 * heads * hd].unflatten(1, (heads, hd))
    v = wide[:, 2 * heads * hd:3 * heads * hd].unflatten(1, (heads, hd))
    slot = torch.randperm(slots, generator=g)[:n].to(torch.int32)
    slot[3], slot[11], slot[20] = -1, slots, 2 ** 31 - 1
    rows = torch.tensor([30, 3, 4, 11, 0, 36, 20, 7, 8], dtype=torch.int32)
    live = 7                                            # the last two of the list are not taken
    ct = torch.uint8 if fp8 else dtype
    fill = 0x31 if fp8 else 3.0
    pool = [torch.full((slots, heads, hd), fill, dtype=ct, device=DEV) for _ in range(2)]
    sc = [torch.full((slots, heads), 127, dtype=torch.uint8, device=DEV) if fp8 else None
          for _ in range(2)]
    kv = B.paged_kv(pool[0], pool[1], page, sc[0], sc[1])
    count = torch.tensor([live], dtype=torch.int32, device=DEV)
    B.paged_store(kv, k, v, slot.to(DEV), rows=rows.to(DEV), n_rows=count)
    written = [r for r in rows[:live].tolist() if 0 <= int(slot[r]) < slots]
    assert len(written) == 4
    rest = torch.ones(slots, dtype=torch.bool)
    for r in written:
        rest[int(slot[r])] = False
    for x, p, s in ((k, pool[0], sc[0]), (v, pool[1], sc[1])):
        p = p.cpu()
        assert (p[rest].float() == fill).all()
        for r in written:
            want = x[r].cpu()
            if fp8:
                val, E = R.quantised(want)
                assert torch.equal(R.e4m3_values()[p[int(slot[r])].long()], val)
                assert torch.equal(s.cpu()[int(slot[r])].long() - 127, E)
            else:
                assert torch.equal(p[int(slot[r])], want)
    # read the whole slot list into rows of a wider tensor; rows behind the count stay
    back = torch.full((n, 2 * heads * hd + 8), 9.0, dtype=dtype, device=DEV)
    ko, vo = (back[:, i * heads * hd:(i + 1) * heads * hd].unflatten(1, (heads, hd)) for i in (0, 1))
    B.paged_load(kv, slot.to(DEV), ko, vo, n_rows=torch.tensor([30], dtype=torch.int32, device=DEV))
    assert (back[30:] == 9.0).all() and (back[:, 2 * heads * hd:] == 9.0).all()
    for o, p, s in ((ko, pool[0], sc[0]), (vo, pool[1], sc[1])):
        for i in range(30):
            at = int(slot[i])
            if not 0 <= at < slots:
                assert (o[i] == 0).all()
                continue
            want = R.cache_values(p.cpu()[at], s.cpu()[at]) if fp8 else p.cpu()[at].double()
            assert torch.equal(o[i].double().cpu(), want)


def test_slots_past_32_bits_of_elements():
    """A cache whose last slots lie past 2^31 elements and 2^32 bytes."""
    heads, hd, page = 32, 256, 64
    slots = (1 << 31) // (heads * hd) + 2 * page
    print(f"paged store and load, {slots} slots of {heads}x{hd}", flush=True)
    pool = [torch.zeros((slots, heads, hd), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    kv = B.paged_kv(pool[0], pool[1], page)
    g = torch.Generator().manual_seed(3)
    x = torch.randn((4, heads, hd), generator=g).to(torch.bfloat16).to(DEV)
    slot = torch.tensor([slots - 1, 0, slots - page, 5], dtype=torch.int32, device=DEV)
    B.paged_store(kv, x, -x, slot)
    ko, vo = torch.empty_like(x), torch.empty_like(x)
    B.paged_load(kv, slot, ko, vo)
    assert torch.equal(ko, x) and torch.equal(vo, -x)
    assert torch.equal(pool[0][slots - 1], x[0])
    assert int(torch.count_nonzero(pool[0][1:5])) == 0


def test_stream_and_graph():
    """On a stream of its own, and captured once and replayed with other values in place."""
    print("paged store and load, captured", flush=True)
    heads, hd, n = 4, 64, 20
    k, v = (torch.randn((n, heads, hd), device=DEV).to(torch.bfloat16) for _ in range(2))
    pool = [torch.zeros((32, heads, hd), dtype=torch.uint8, device=DEV) for _ in range(2)]
    sc = [torch.zeros((32, heads), dtype=torch.uint8, device=DEV) for _ in range(2)]
    kv = B.paged_kv(pool[0], pool[1], 8, sc[0], sc[1])
    slot = torch.randperm(32, device=DEV)[:n].to(torch.int32)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.paged_store(kv, k, v, slot)
        B.paged_load(kv, slot, ko, vo)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.paged_store(kv, k, v, slot)
        B.paged_load(kv, slot, ko, vo)
    for _ in range(3):
        k.copy_(torch.randn((n, heads, hd), device=DEV))
        v.copy_(torch.randn((n, heads, hd), device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        for x, o in ((k, ko), (v, vo)):
            val, E = R.quantised(x.cpu())
            assert torch.equal(o.double().cpu(), val * R.power(E).unsqueeze(-1))
