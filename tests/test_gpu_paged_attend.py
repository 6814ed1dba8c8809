"""adept_paged_attend against the definition in 64 bits (tests/paged_ref.py gives the tolerances)."""
import math
import random

import pytest
import torch

from paper_2601_03700_amd import binding as B
from tests import paged_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Case:
    """Entries and a cache.  shape: per sequence (earlier tokens, new tokens, share of the new
    ones that is active); junk: what every slot holds that no entry may read."""

    def __init__(self, dt, cache, H, heads, hd, page, shape, seed=1, junk=math.nan, spare=3,
                 q_std=1.5):
        self.dt, self.H, self.hd, self.page, self.heads = R.TDT[dt], H, hd, page, heads
        r = random.Random(seed)
        g = torch.Generator().manual_seed(seed)
        lens = [c + n for c, n, _ in shape]
        need = [-(-n // page) for n in lens]
        total = sum(need) + spare
        order = torch.randperm(total, generator=g).tolist()
        self.n_seq = len(shape)
        self.table = torch.full((self.n_seq, max(max(need), 1)), -1, dtype=torch.int32)
        filled = torch.zeros(total * page, dtype=torch.bool)
        for b, m in enumerate(need):
            mine, order = order[:m], order[m:]
            self.table[b, :m] = torch.tensor(mine, dtype=torch.int32)
            for t in range(lens[b]):
                filled[mine[t // page] * page + t % page] = True
        pos, seq, rows = [], [], []
        for b, (c, n, share) in enumerate(shape):
            live = sorted(r.sample(range(n), round(share * n)))
            rows += [len(pos) + j for j in live]
            pos += range(c, c + n)
            seq += [b] * n
        self.pos, self.seq = (torch.tensor(x, dtype=torch.int32) for x in (pos, seq))
        self.rows = torch.tensor(rows, dtype=torch.int32)
        slots = total * page
        wide = 1 + 3 * (torch.rand((heads, hd), generator=g) < 0.05)
        x = [torch.randn((slots, heads, hd), generator=g) * wide for _ in range(2)]
        self.scales = [None, None]
        if cache == "fp8":
            codes = [(t / 0.125).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for t in x]
            self.scales = [torch.randint(122, 126, (slots, heads), generator=g).to(torch.uint8)
                           for _ in x]
            self.pool = codes
            for p in self.pool:
                p[~filled] = 0x7f if math.isnan(junk) else 0x7e
        else:
            self.pool = [t.to(R.TDT[cache]) for t in x]
            for p in self.pool:
                p[~filled] = junk
        self.q = (torch.randn((len(rows), H, hd), generator=g) * q_std).to(self.dt)
        self.live = self.key_len = None
        self.causal = True
        self.scale = 1 / math.sqrt(hd)

    def values(self):
        if self.scales[0] is None:
            return [p.to(DEV) for p in self.pool]
        return [R.cache_values(p, s).to(DEV) for p, s in zip(self.pool, self.scales)]

    def run(self, max_active=None, out=None, stream=None):
        d = lambda t: None if t is None else t.to(DEV)
        n = len(self.rows)
        m = n if max_active is None else max_active
        kv = B.paged_kv(d(self.pool[0]), d(self.pool[1]), self.page, d(self.scales[0]),
                        d(self.scales[1]))
        q = torch.zeros((m, self.H, self.hd), dtype=self.dt, device=DEV)
        q[:n] = self.q.to(DEV)
        rows = torch.full((m,), -7, dtype=torch.int32, device=DEV)      # behind the count: not read
        rows[:n] = self.rows.to(DEV)
        out = torch.full_like(q, 7.0) if out is None else out
        ws = torch.randint(0, 256, (B.paged_attend_workspace_bytes(
            kv, self.H, m, self.n_seq, self.table.shape[1]),), dtype=torch.uint8, device=DEV)
        B.paged_attend(kv, q, rows, torch.tensor([n], dtype=torch.int32, device=DEV), m,
                       d(self.pos), d(self.seq), self.n_seq, d(self.table), out, causal=self.causal,
                       key_len=d(self.key_len), key_live=d(self.live), workspace=ws,
                       scale=self.scale)
        assert (out[n:] == 7.0).all()
        return out[:n]

    def ref(self):
        at = self.rows.long()
        k, v = self.values()
        return R.attend(self.q.to(DEV), k, v, self.table.to(DEV), self.page, self.pos[at],
                        self.seq[at], self.scale, self.causal, self.key_len,
                        None if self.live is None else self.live.to(DEV))

    def check(self, **kw):
        out = self.run(**kw)
        ref, wv, qk = self.ref()
        seen = torch.isfinite(ref)          # an entry that sees NaN has no other result
        assert torch.equal(torch.isfinite(out), seen)
        err = (out.double() - ref).abs()
        worst = (err / R.bound(self.dt, ref, wv, qk))[seen].max().item()
        print(f"  worst error / bound {worst:.3f}", flush=True)
        assert worst <= 1.0
        return out


TYPES = [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32"), ("f32", "fp8")]
HEADS = [(2, 2, 128), (5, 5, 64), (8, 2, 128), (6, 2, 64), (16, 1, 64), (40, 1, 128), (3, 3, 32),
         (4, 2, 256), (2, 2, 16)]
SHAPES = {
    "one token": [(0, 1, 1)],
    "decode": [(0, 1, 1), (1, 1, 1), (62, 1, 1), (63, 1, 1), (64, 1, 1), (300, 1, 1)],
    "long decode": [(2500, 1, 1)],
    "short chunks": [(5, 3, 1), (0, 2, 1), (131, 7, 1)],
    "chunks": [(0, 64, 1), (33, 65, 1), (200, 129, 0.7), (7, 1, 1)],
    "prompt": [(0, 257, 1)],
}


@pytest.mark.parametrize("dt,cache", TYPES)
@pytest.mark.parametrize("H,heads,hd", HEADS)
@pytest.mark.parametrize("shape", SHAPES)
def test_matches_definition(dt, cache, H, heads, hd, shape):
    page = {"one token": 1, "decode": 16, "long decode": 64, "short chunks": 4, "chunks": 32,
            "prompt": 128}[shape]
    print(f"paged attend {dt}/{cache} {H}/{heads}x{hd} {shape}", flush=True)
    Case(dt, cache, H, heads, hd, page, SHAPES[shape]).check()


@pytest.mark.parametrize("dt,cache", TYPES)
@pytest.mark.parametrize("page", [1, 2, 8, 16, 64, 256, 1024])
def test_pages(dt, cache, page):
    """Pages smaller and larger than a tile, ending inside one; a bound above the count."""
    print(f"paged attend, pages of {page}, {dt}/{cache}", flush=True)
    Case(dt, cache, 4, 2, 64, page, [(90, 30, 1), (0, 200, 0.5), (517, 1, 1)], seed=page).check(
        max_active=400)
    Case(dt, cache, 4, 4, 128, page, [(90, 1, 1), (700, 1, 1), (0, 1, 1)], seed=page).check(
        max_active=3)


@pytest.mark.parametrize("dt,cache", TYPES)
@pytest.mark.parametrize("chunk", [1, 70])
def test_many_sequences(dt, cache, chunk):
    """More sequences than a wave has lanes, lengths all over, some without any entry."""
    print(f"paged attend, 150 sequences, {dt}/{cache} chunk={chunk}", flush=True)
    r = random.Random(3)
    shape = [(r.choice([0, 3, 50, 129, 400]), r.randint(1, chunk), r.choice([0, 0.5, 1, 1]))
             for _ in range(150)]
    Case(dt, cache, 4, 2, 64, 16, shape).check(max_active=max(150, 150 * chunk // 2))


@pytest.mark.parametrize("dt,cache", TYPES)
@pytest.mark.parametrize("H,heads,hd", [(4, 2, 64), (2, 2, 128), (2, 1, 256)])
@pytest.mark.parametrize("shape", [[(100, 1, 1), (700, 1, 1), (40, 1, 1), (200, 1, 1)],
                                   [(100, 40, 1), (0, 150, 1), (30, 5, 1), (200, 3, 1)]])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("past_end", [True, False])
def test_masks(dt, cache, H, heads, hd, shape, causal, past_end):
    """Key lengths (0 and negative among them), dead slots, pages that are not there, sequences
    outside the table: rows with nothing to see are zeros, and what is left out holds NaN."""
    print(f"paged attend, masks {dt}/{cache} {H}/{heads}x{hd} causal={causal} {shape}", flush=True)
    c = Case(dt, cache, H, heads, hd, 16, shape, seed=4)
    c.causal = causal
    g = torch.Generator().manual_seed(1)
    c.live = (torch.rand(c.pool[0].shape[0], generator=g) < 0.7).to(torch.uint8) * 3
    c.live[c.table[2][c.table[2] >= 0].long()[:, None] * 16 + torch.arange(16)] = 0   # all of it
    for p in c.pool:
        p[c.live == 0] = 0x7f if cache == "fp8" else math.nan
    c.table[0, 1], c.table[0, 3] = c.pool[0].shape[0] // 16, -2 ** 31
    c.table[1, 0] = 2 ** 31 - 1
    # past_end: lengths that take in the slots behind a sequence's last token
    ends = [10 ** 6] * 2 if past_end else [ctx + new for ctx, new, _ in shape[1:3]]
    c.key_len = torch.tensor([90, *ends, 0 if causal else -5], dtype=torch.int32)
    out = c.check()
    at = c.seq[c.rows.long()]
    assert (out[at.to(DEV) >= 2] == 0).all()
    c.seq = torch.where(c.seq == 1, torch.tensor(4, dtype=torch.int32), c.seq)
    c.seq[0] = -1
    c.check()


@pytest.mark.parametrize("dt,cache", TYPES)
@pytest.mark.parametrize("H,heads,hd", [(4, 2, 64), (2, 2, 128)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_later_tokens_do_not_reach_earlier_ones(dt, cache, H, heads, hd, bad):
    """A token of the chunk whose K and V are NaN or infinite: entries before it are as if it were
    zeros, entries that see it are not finite, and other sequences are not touched."""
    print(f"paged attend, {bad} in a chunk, {dt}/{cache} {H}/{heads}x{hd}", flush=True)
    shape = [(60, 100, 1), (10, 90, 1), (200, 1, 1)]
    c = Case(dt, cache, H, heads, hd, 16, shape, seed=6)
    clean = c.check()
    t = 97                                              # of sequence 0
    slot = int(c.table[0, t // 16]) * 16 + t % 16
    for p in c.pool[1:] if math.isinf(bad) else c.pool:
        p[slot] = 0x7f if cache == "fp8" else bad
    got = c.run()
    at = c.rows.long()
    sees = ((c.seq[at] == 0) & (c.pos[at] >= t)).to(DEV)
    ref = c.ref()
    err = (got[~sees].double() - ref[0][~sees]).abs()
    assert (err <= R.bound(c.dt, *ref)[~sees]).all()
    assert not torch.isfinite(got[sees]).any()
    assert sees.sum() == 160 - t and torch.isfinite(clean).all()


@pytest.mark.parametrize("dt,cache", [("bf16", "bf16"), ("f32", "f32")])
def test_order_of_entries_and_positions(dt, cache):
    """Entries in any order, one of them twice, positions that fall and are negative."""
    print(f"paged attend, entries in any order {dt}", flush=True)
    c = Case(dt, cache, 4, 2, 64, 8, [(40, 30, 1), (0, 50, 1), (9, 20, 1)], seed=8)
    g = torch.Generator().manual_seed(2)
    perm = torch.randperm(100, generator=g)
    perm[7] = perm[3]
    c.rows, c.q = c.rows[perm], c.q[perm]
    c.pos[int(c.rows[5])] = -3
    c.pos[int(c.rows[6])] = 2 ** 31 - 1                 # everything there is
    out = c.check()
    assert (out[5] == 0).all()


@pytest.mark.parametrize("dt,cache", TYPES)
@pytest.mark.parametrize("chunk", [1, 40])
def test_large_scores(dt, cache, chunk):
    """Scores of some hundreds: the running maximum has to move, weights underflow."""
    print(f"paged attend, large scores {dt}/{cache} chunk={chunk}", flush=True)
    Case(dt, cache, 4, 2, 64, 16, [(300, chunk, 1), (5, chunk, 1)], seed=9, q_std=60.0).check()


@pytest.mark.parametrize("dt,cache", TYPES)
def test_long_context(dt, cache):
    """A long context for few entries, whose page table and keys are cut into many pieces."""
    print(f"paged attend, long context {dt}/{cache}", flush=True)
    Case(dt, cache, 8, 2, 64, 64, [(40000, 1, 1), (3, 1, 1)], seed=11).check()
    Case(dt, cache, 8, 2, 64, 64, [(20000, 5, 1), (3, 2, 1)], seed=12).check()


@pytest.mark.parametrize("chunk", [1, 20])
def test_slots_past_32_bits_of_bytes(chunk):
    """The keys' slots lie past 2^32 bytes of the cache."""
    H, heads, hd, page = 32, 32, 128, 64
    slots = (1 << 32) // (heads * hd * 2) + 8 * page
    print(f"paged attend, {slots} slots, chunk={chunk}", flush=True)
    pool = [torch.zeros((slots, heads, hd), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    n_pages = slots // page
    table = torch.tensor([[n_pages - 1, 0, n_pages - 3]], dtype=torch.int32, device=DEV)
    for p in table[0].tolist():
        for x in pool:
            x[p * page:(p + 1) * page] = torch.randn((page, heads, hd), device=DEV)
    q = torch.randn((chunk, H, hd), device=DEV).to(torch.bfloat16)
    pos = torch.arange(150 - chunk, 150, dtype=torch.int32, device=DEV)
    seq = torch.zeros_like(pos)
    rows = torch.arange(chunk, dtype=torch.int32, device=DEV)
    kv = B.paged_kv(pool[0], pool[1], page)
    ws = torch.empty(B.paged_attend_workspace_bytes(kv, H, chunk, 1, 3), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    B.paged_attend(kv, q, rows, torch.tensor([chunk], dtype=torch.int32, device=DEV), chunk, pos,
                   seq, 1, table, out, workspace=ws)
    ref, wv, qk = R.attend(q, pool[0], pool[1], table, page, pos, seq, 1 / math.sqrt(hd))
    assert ((out.double() - ref).abs() <= R.bound(torch.bfloat16, ref, wv, qk)).all()


@pytest.mark.parametrize("dt,cache", TYPES)
@pytest.mark.parametrize("chunk", [1, 33])
def test_same_bits_each_time_and_in_a_graph(dt, cache, chunk):
    """Eager, again, on another stream, and replayed: the same bits; two graphs that share a
    workspace, replayed in turn."""
    print(f"paged attend, captured {dt}/{cache} chunk={chunk}", flush=True)
    cases = [Case(dt, cache, 8, 2, 128, 16, [(900, chunk, 1), (70, chunk, 1)], seed=s) for s in (1, 2)]
    calls, ws = [], torch.empty(64 << 20, dtype=torch.uint8, device=DEV)
    for c in cases:
        want = c.run()
        d = lambda t: None if t is None else t.to(DEV)
        kv = B.paged_kv(d(c.pool[0]), d(c.pool[1]), 16, d(c.scales[0]), d(c.scales[1]))
        args = [d(c.q), d(c.rows), torch.tensor([len(c.rows)], dtype=torch.int32, device=DEV),
                len(c.rows), d(c.pos), d(c.seq), 2, d(c.table), torch.empty_like(d(c.q))]
        need = B.paged_attend_workspace_bytes(kv, 8, len(c.rows), 2, c.table.shape[1])
        assert need <= ws.numel()
        calls.append((kv, args, want))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    for kv, args, want in calls:
        B.paged_attend(kv, *args, workspace=ws)
        assert torch.equal(args[-1], want)
        torch.cuda.synchronize()
        B.paged_attend(kv, *args, workspace=ws, stream=s)
        s.synchronize()
        assert torch.equal(args[-1], want)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.paged_attend(kv, *args, workspace=ws)
        graphs.append(g)
    for _ in range(3):
        for (kv, args, want), g in zip(calls, graphs):
            args[-1].fill_(5.0)
            ws.random_(0, 255)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(args[-1], want)
        B.paged_attend(calls[0][0], *calls[0][1], workspace=ws)
        torch.cuda.synchronize()


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("shape", [[(900, 33, 1), (70, 33, 1)], [(300, 33, 1)],
                                   [(900, 1, 1), (70, 1, 1), (5, 1, 1)]])
def test_the_same_bits_ten_times(cache, hd, shape):
    """Nothing left over in registers or LDS enters a result, the choice of the softmax's
    reference among it."""
    print(f"paged attend, ten times, bf16/{cache} hd={hd} {shape}", flush=True)
    c = Case("bf16", cache, 8, 2, hd, 16, shape, seed=2)
    first = c.check()
    for _ in range(10):
        assert torch.equal(c.run(), first)


def test_chunks_are_written_and_attended_in_turn():
    """A prompt in pieces of different lengths through the 8-bit and the bf16 cache, then single
    tokens, as a program runs it: each step's rows are stored, then attended with, and the cache
    read back at the end holds what was stored."""
    print("paged cache: store, attend, load in turn", flush=True)
    H, heads, hd, page, n_seq = 8, 2, 64, 8, 3
    for dt, cache in (("bf16", "bf16"), ("bf16", "fp8"), ("f32", "fp8")):
        dtype = R.TDT[dt]
        steps = [[50, 3, 17], [1, 30, 9], [70, 1, 1], [1, 1, 1], [1, 1, 1]]
        total = [sum(s[b] for s in steps) for b in range(n_seq)]
        pages = [-(-t // page) for t in total]
        g = torch.Generator().manual_seed(1)
        order = torch.randperm(sum(pages) + 2, generator=g).to(torch.int32)
        table = torch.full((n_seq, max(pages)), -1, dtype=torch.int32)
        for b in range(n_seq):
            table[b, :pages[b]] = order[sum(pages[:b]):sum(pages[:b + 1])]
        slots = order.numel() * page
        ct = torch.uint8 if cache == "fp8" else dtype
        pool = [torch.full((slots, heads, hd), 0x7f, dtype=ct, device=DEV) for _ in range(2)]
        sc = [torch.zeros((slots, heads), dtype=torch.uint8, device=DEV) if cache == "fp8" else None
              for _ in range(2)]
        kv = B.paged_kv(pool[0], pool[1], page, sc[0], sc[1])
        tab = table.to(DEV)
        ref = [torch.zeros((slots, heads, hd), dtype=torch.float64) for _ in range(2)]
        done = [0] * n_seq
        for step in steps:
            pos = torch.tensor([done[b] + j for b in range(n_seq) for j in range(step[b])])
            seq = torch.tensor([b for b in range(n_seq) for _ in range(step[b])])
            slot = table[seq, pos // page].long() * page + pos % page
            n = len(pos)
            q = torch.randn((n, H, hd), generator=g).to(dtype)
            k, v = (torch.randn((n, heads, hd), generator=g).to(dtype) for _ in range(2))
            for x, r in ((k, ref[0]), (v, ref[1])):
                val, E = R.quantised(x)
                r[slot] = val * R.power(E).unsqueeze(-1) if cache == "fp8" else x.double()
            i32 = lambda t: t.to(torch.int32).to(DEV)
            B.paged_store(kv, k.to(DEV), v.to(DEV), i32(slot))
            out = torch.empty_like(q, device=DEV)
            ws = torch.empty(B.paged_attend_workspace_bytes(kv, H, n, n_seq, table.shape[1]),
                             dtype=torch.uint8, device=DEV)
            B.paged_attend(kv, q.to(DEV), i32(torch.arange(n)), i32(torch.tensor([n])), n, i32(pos),
                           i32(seq), n_seq, tab, out, workspace=ws)
            want = R.attend(q, ref[0], ref[1], table, page, pos, seq, 1 / math.sqrt(hd))
            err = (out.double().cpu() - want[0]).abs()
            assert (err <= R.bound(dtype, *want)).all()
            done = [d + s for d, s in zip(done, step)]
        t = torch.cat([torch.arange(n) for n in total])
        b = torch.cat([torch.full((n,), i) for i, n in enumerate(total)])
        slot = table[b, t // page].long() * page + t % page
        ko, vo = (torch.empty((len(t), heads, hd), dtype=dtype, device=DEV) for _ in range(2))
        B.paged_load(kv, slot.to(torch.int32).to(DEV), ko, vo)
        assert torch.equal(ko.double().cpu(), ref[0][slot])
        assert torch.equal(vo.double().cpu(), ref[1][slot])


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("n,bound", [(1025, 1025), (1500, 1500), (1024, 1500), (3, 1500), (0, 1500)])
def test_long_lists_of_single_tokens(cache, n, bound):
    """More entries than the cut of long ones counts, and a bound above it with fewer there."""
    print(f"paged attend, {n} of {bound} single tokens, {cache}", flush=True)
    lens = [(17 * i) % 90 for i in range(bound)]
    if 0 < n < 10:
        lens[0] = 3000
    c = Case("bf16", cache, 2, 1, 64, 16, [(t, 1, 1) for t in lens], seed=n)
    c.rows, c.q = c.rows[:n], c.q[:n]
    c.check(max_active=bound) if n else c.run(max_active=bound)


@pytest.mark.parametrize("dt,cache", [("bf16", "fp8"), ("f32", "f32")])
def test_long_lists_of_chunks(dt, cache):
    """More entries than one pass of the plan takes, more sequences than a wave has lanes, with
    one to four tiles each."""
    print(f"paged attend, 9000 entries, {dt}/{cache}", flush=True)
    shape = [(3 * b, 30 + (37 * b) % 190, 1) for b in range(72)]
    c = Case(dt, cache, 2, 1, 64, 32, shape)
    assert len(c.rows) > 8192
    c.check(max_active=len(c.rows) + 500)


@pytest.mark.parametrize("n_seq", [1023, 1024, 1025, 1200])
def test_many_sequences_of_two_tokens(n_seq):
    """Hundreds of short tiles in one call."""
    print(f"paged attend, {n_seq} sequences of 2 tokens", flush=True)
    Case("bf16", "bf16", 2, 1, 64, 16, [((5 * b) % 40, 2, 1) for b in range(n_seq)]).check()


@pytest.mark.parametrize("chunk", [1, 40])
def test_two_calls_at_once(chunk):
    """On two streams, each with its workspace: the bits of the calls alone."""
    print(f"paged attend, two streams, {chunk}", flush=True)
    cases = [Case("bf16", kind, 4, 2, 128, 16, [(900, chunk, 1), (70, chunk, 1)], seed=s)
             for s, kind in ((1, "bf16"), (2, "fp8"))]
    alone = [c.run().clone() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    out = [[], []]
    for _ in range(5):
        for i, c in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                out[i].append(c.run())
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, alone[i]) for x in out[i])
