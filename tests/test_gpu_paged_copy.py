"""adept_paged_copy: pages of all layers, whole or their first tokens, bit for bit."""
import pytest
import torch

from paper_2601_03700_amd import binding as B

pytestmark = pytest.mark.gpu


def pool(kind, layers, pages, page, heads, hd, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dims = (layers, pages * page, heads, hd)
    size = {"f32": 4, "bf16": 2, "fp8": 1}[kind]
    make = lambda shape: torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8)
    out = {}
    for tag in ("k", "v"):
        raw = make((layers, pages * page, heads, hd * size))      # any bits, NaN among them
        out[tag] = raw if kind == "fp8" else raw.view(torch.float32 if kind == "f32" else torch.bfloat16)
        assert out[tag].shape == dims
        if kind == "fp8":
            out[tag + "_scale"] = make(dims[:3])
    return out


def handle(p, page):
    return B.paged_kv(p["k"][0], p["v"][0], page, *((p["k_scale"][0], p["v_scale"][0])
                                                    if "k_scale" in p else (None, None)))


def bits(t):
    return t.view(torch.uint8) if t.dtype != torch.uint8 else t


def expect(p, page, n_pages, layers, src, dst, count, n):
    out = {tag: bits(t).clone() for tag, t in p.items()}
    for i in range(n):
        s, d = src[i], dst[i]
        if not (0 <= s < n_pages and 0 <= d < n_pages):
            continue
        m = page if count is None else min(max(count[i], 0), page)
        for tag in p:
            out[tag][:layers, d * page:d * page + m] = bits(p[tag])[:layers, s * page:s * page + m]
    return out


@pytest.mark.parametrize("kind", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("heads,hd,page", [(1, 16, 1), (2, 64, 16), (25, 64, 8), (8, 128, 64),
                                           (3, 256, 4), (1, 32, 1024)])
def test_pages(kind, heads, hd, page):
    layers, n_pages = 3, 11
    p = pool(kind, layers, n_pages, page, heads, hd)
    kv = handle(p, page)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    for src, dst, count in [([4], [9], None), ([0, 4, 0, 10], [1, 2, 3, 5], None),
                            ([0, 4, 0, 10, 6], [1, 2, 3, 5, 9], [0, page, 1, -3, page + 7]),
                            ([-1, 11, 4, 7], [2, 3, 1 << 30, 0], None), ([], [], None)]:
        want = expect(p, page, n_pages, layers, src, dst, count, len(src))
        B.paged_copy(kv, layers, i32(src), i32(dst), None if count is None else i32(count))
        for tag in p:
            assert torch.equal(bits(p[tag]), want[tag]), tag


def test_a_count_on_the_device_and_fewer_layers():
    p = pool("fp8", 4, 9, 16, 5, 32)
    kv = handle(p, 16)
    src, dst = [0, 1, 2], [6, 7, 8]
    for live in (0, 2, 3, 50, -1):
        want = expect(p, 16, 9, 2, src, dst, None, max(0, min(live, 3)))
        B.paged_copy(kv, 2, *(torch.tensor(x, dtype=torch.int32, device="cuda") for x in (src, dst)),
                     n_pages=torch.tensor([live], dtype=torch.int32, device="cuda"))
        for tag in p:
            assert torch.equal(p[tag], want[tag]), (tag, live)


def test_far_pages_of_a_large_cache():
    """Offsets behind 2^32 bytes."""
    page, heads, hd, pages = 64, 32, 128, 9000             # 4.7 GB each of K and V
    p = {tag: torch.zeros((1, pages * page, heads, hd), dtype=torch.bfloat16, device="cuda")
         for tag in ("k", "v")}
    for i, s in enumerate((8191, 8999)):
        p["k"][0, s * page:(s + 1) * page] = i + 1
        p["v"][0, s * page:(s + 1) * page] = -i - 1
    kv = handle(p, page)
    B.paged_copy(kv, 1, *(torch.tensor(x, dtype=torch.int32, device="cuda")
                          for x in ([8191, 8999], [8998, 1])))
    for d, v in ((8998, 1), (1, 2)):
        assert (p["k"][0, d * page:(d + 1) * page] == v).all()
        assert (p["v"][0, d * page:(d + 1) * page] == -v).all()
    assert int((p["k"] != 0).sum()) == 4 * page * heads * hd
