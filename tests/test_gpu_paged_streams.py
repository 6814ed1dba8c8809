"""Two calls of adept_paged_attend that run at the same time."""
import pytest
import torch

from paper_2601_03700_amd import binding as B
from tests.test_gpu_paged_attend import Case

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("chunk", [1, 150])
def test_two_streams_filled_before_either_runs(chunk):
    """Everything is on the device beforehand, each call has its own workspace, and both streams
    wait for the same event until their calls are queued: the bits of the calls alone."""
    print(f"paged attend, two filled streams, chunk={chunk}", flush=True)
    d = lambda t: None if t is None else t.to(DEV)
    calls = []
    for seed, kind in ((1, "bf16"), (2, "fp8")):
        c = Case("bf16", kind, 8, 4, 128, 64, [(5000, chunk, 1), (1300, chunk, 1), (4000, chunk, 1)],
                 seed=seed)
        want = c.check().clone()
        kv = B.paged_kv(d(c.pool[0]), d(c.pool[1]), 64, d(c.scales[0]), d(c.scales[1]))
        n = len(c.rows)
        args = [d(c.q), d(c.rows), torch.tensor([n], dtype=torch.int32, device=DEV), n, d(c.pos),
                d(c.seq), 3, d(c.table)]
        ws = torch.empty(B.paged_attend_workspace_bytes(kv, 8, n, 3, c.table.shape[1]),
                         dtype=torch.uint8, device=DEV)
        outs = [torch.full_like(args[0], 7.0) for _ in range(8)]
        calls.append((kv, args, ws, outs, want, torch.cuda.Stream()))
    big = torch.zeros(1 << 30, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    for _ in range(8):                   # some milliseconds in which the calls are queued
        big.copy_(big.roll(1))
    go = torch.cuda.Event()
    go.record()
    for *_, s in calls:
        s.wait_event(go)
    for i in range(8):
        for kv, args, ws, outs, _, s in calls:
            B.paged_attend(kv, *args, outs[i], workspace=ws, stream=s)
    torch.cuda.synchronize()
    for _, _, _, outs, want, _ in calls:
        for out in outs:
            assert torch.equal(out, want)
