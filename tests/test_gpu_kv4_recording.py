"""Calls on a stream that is being recorded into a graph: what would write block tables is refused and changes nothing, for a replay
would write them again when the blocks may be another client's."""
import pytest
import torch

from paper_2605_13319_amd import nav
from tests.test_gpu_kv4 import make_cache, random_rows, refused, shape_of

pytestmark = pytest.mark.gpu

NQ, NKV, DIM = 8, 2, 64


def rows(n, seed):
    return random_rows(n, NKV, DIM, "bf16", seed).cuda()


def test_new_blocks_and_cuts_are_refused():
    kv = make_cache(shape_of(NQ, NKV, DIM), 3, 64)
    kv.extend([0, 1], [40, 20])
    k = rows(60, 1)
    kv.append(0, k, k)
    kv.extend([0], [2])
    new = rows(2, 2)
    q, out = random_rows(2, NQ, DIM, "bf16", 3).cuda(), torch.zeros(2, NQ, DIM, dtype=torch.bfloat16, device="cuda")
    mass = torch.rand(3, 1, NKV, 64, device="cuda")
    kv.append(0, new, new)
    want = kv.attend(0, q).clone()
    torch.cuda.synchronize()
    state = [kv.length(c) for c in range(3)], [kv.seq_blocks(c) for c in range(3)], kv.free_blocks()
    kept = torch.zeros(1, 1, NKV, 10, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for f in (lambda: kv.extend([0, 2], [2, 1]), lambda: kv.extend([0], [7]), lambda: kv.extend([1], [20]),
                  lambda: kv.evict([1], [1], 10, 2, mass, kept=kept), lambda: kv.evict([1], [2], 10, 2, mass, kept=kept)):
            refused(nav.ESTATE, f)
        assert state == ([kv.length(c) for c in range(3)], [kv.seq_blocks(c) for c in range(3)], kv.free_blocks())
        kv.append(0, new, new)  # (the pass goes on)
        kv.attend(0, q, out=out)
    for _ in range(3):
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    # what was refused is right afterwards: the entries have not been taken for written
    kv.extend([0, 2], [7, 30])
    new = rows(37, 4)
    kv.append(0, new, new)
    got = kv.read([2, 0], [0, 42], [30, 7])[0][0]
    kv.truncate([0, 2], [0, 0])
    kv.extend([0], [37])
    kv.append(0, new, new)
    again = kv.read([0], [0], [37])[0][0]
    assert torch.equal(got, torch.cat([again[7:], again[:7]]))


def test_a_whole_round_is_recorded_where_no_block_is_new():
    """Rows taken back and asked for again, behind the same blocks: nothing to write."""
    kv = make_cache(shape_of(NQ, NKV, DIM), 1, 64)
    kv.extend([0], [17])
    kv.append(0, rows(17, 1), rows(17, 2))
    new = rows(5, 3)
    q, out = random_rows(5, NQ, DIM, "bf16", 4).cuda(), torch.zeros(5, NQ, DIM, dtype=torch.bfloat16, device="cuda")
    kv.extend([0], [5])
    kv.append(0, new, new)
    kv.attend(0, q)
    kv.truncate([0], [17])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv.extend([0], [5])
        kv.append(0, new, new)
        kv.attend(0, q, out=out)
    for seed in range(3):
        new.copy_(rows(5, 10 + seed))
        q.copy_(random_rows(5, NQ, DIM, "bf16", 20 + seed).cuda())
        kv.append(0, new, new)
        want = kv.attend(0, q).clone()
        new_was = new.clone()
        kv.append(0, new * 2, new * 2)
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(new, new_was)
