"""A recorded attention goes on working when a larger pass has made the handle's scratch grow: the memory that it was recorded with is
kept.  (Without that a replay reads and writes memory that has been given back; these tests run only on code that keeps it.)"""
import pytest
import torch

from tests.test_gpu_kv4 import make_cache, random_rows, shape_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,before", [((8, 2, 64), 3000), ((32, 8, 128), 700)])
def test_replays_after_the_scratch_has_grown(heads, before, dtype):
    nq, nkv, dim = heads
    kv = make_cache(shape_of(*heads, dtype), 1, before + 2100)
    x = random_rows(before, nkv, dim, dtype, 1).cuda()
    kv.extend([0], [before])
    kv.append(0, x, x)
    new = random_rows(5, nkv, dim, dtype, 2).cuda()
    kv.extend([0], [5])
    kv.append(0, new, new)
    q = random_rows(5, nq, dim, dtype, 3).cuda()
    out, mass = torch.zeros_like(q), torch.zeros(1, 1, nkv, before + 2100, device="cuda")
    kv.attend(0, q, out=out, mass=mass, decay=0.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv.attend(0, q, out=out, mass=mass, decay=0.0)
    for grown in (40, 333, 2048):  # each takes more scratch than the one before
        kv.truncate([0], [before])
        kv.extend([0], [grown])
        rows = random_rows(grown, nkv, dim, dtype, 4).cuda()
        kv.append(0, rows, rows)
        kv.attend(0, random_rows(grown, nq, dim, dtype, 5).cuda(), mass=torch.zeros_like(mass), decay=0.0)
        kv.truncate([0], [before])
        kv.extend([0], [5])
        kv.append(0, new, new)
        q.copy_(random_rows(5, nq, dim, dtype, 10 + grown))
        other = torch.zeros_like(mass)
        want = kv.attend(0, q, mass=other, decay=0.0)
        torch.full((1 << 24,), float("nan"), device="cuda").sum().item()  # (memory that is free would be written over)
        for _ in range(2):
            out.fill_(7)
            mass.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(mass[..., :before + 5], other[..., :before + 5])
