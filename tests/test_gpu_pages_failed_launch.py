"""A launch that is said to have failed (here: an error that an earlier call of the process left behind is taken for its own): the clients hold
what they held, on the device as well, whoever gets the blocks that were given back."""
import ctypes as C

import pytest
import torch

from paper_2605_13319_amd import nav
from tests.test_gpu_pages import make_cache, random_rows, shape_of

gpu = pytest.mark.gpu
NKV, DIM = 2, 64


def leave_an_error():
    with open("/proc/self/maps") as f:
        path = next(line.split()[-1] for line in f if "libamdhip64" in line)
    assert C.CDLL(path).hipSetDevice(4096) != 0  # (no such device: nothing else happens)


def ints(*x):
    return (C.c_int32 * len(x))(*x)


def failed(pg, call, *args):
    torch.cuda.synchronize()
    leave_an_error()
    assert call(pg.handle, *args, pg._stream()) == nav.EHIP


def rows(n, seed):
    return random_rows(n, NKV, DIM, "bf16", seed).cuda()


def begun():
    """Client 1 holds client 0's 21 tokens, in the same blocks; client 3 is in a pass of a tree."""
    pg = make_cache(shape_of(4, NKV, DIM), 5, 40)
    x = rows(21, 1)
    pg.extend([0], [21])
    pg.append(0, x, x)
    pg.fork([0], [1])
    pg.extend([3], [3], [-1, 0, 0])
    pg.append(0, rows(3, 2), rows(3, 2))
    return pg, x


def others_write(pg):
    n = pg.free_blocks() * 16
    pg.extend([4], [n])
    pg.append(0, rows(n, 9), rows(n, 9))


@gpu
def test_clients_keep_their_text_when_a_pass_could_not_begin():
    pg, x = begun()
    free = pg.free_blocks()
    failed(pg, nav._lib.pipesd_pages_extend, 2, ints(1, 2), ints(2, 5), ints(-1, 0, -1, 0, 0, 1, 1))
    assert pg.free_blocks() == free and [pg.length(c) for c in range(4)] == [21, 21, 0, 3]
    with pytest.raises(nav.PipesdError) as e:  # (its trees are not the pass's any more)
        pg.attend(0, random_rows(3, 4, DIM, "bf16", 3).cuda())
    assert e.value.status == nav.ESTATE
    others_write(pg)
    for c in (0, 1):
        assert torch.equal(pg.read([c], [0], [21])[0][0], x)
    pg.truncate([4], [0])
    y = rows(2, 5)
    pg.extend([1], [2])
    pg.append(0, y, y)
    assert torch.equal(pg.read([1], [0], [23])[0][0], torch.cat([x, y])) and torch.equal(pg.read([0], [0], [21])[0][0], x)


@gpu
@pytest.mark.parametrize("name", ["fork", "copy"])
def test_targets_are_empty_when_they_could_not_become_a_copy(name):
    pg, x = begun()
    free = pg.free_blocks() + 1
    failed(pg, getattr(nav._lib, "pipesd_pages_" + name), 2, ints(0, 1), ints(2, 3), ints(20, 21))
    assert pg.free_blocks() == free and [pg.length(c) for c in range(4)] == [21, 21, 0, 0]
    others_write(pg)
    for c in (0, 1):
        assert torch.equal(pg.read([c], [0], [21])[0][0], x)
    pg.truncate([4], [0])
    getattr(pg, name)([0, 1], [2, 3], [20, 21])
    assert torch.equal(pg.read([2, 3], [0, 0], [20, 21])[0][0], torch.cat([x[:20], x]))


@gpu
def test_blocks_that_others_hold_are_not_written_by_a_compaction_that_could_not_run():
    pg, x = begun()
    free = pg.free_blocks()
    failed(pg, nav._lib.pipesd_pages_compact, 1, ints(1), ints(2), ints(3), ints(1, 2, 18))
    assert pg.free_blocks() == free and pg.length(1) == 21
    others_write(pg)
    for c in (0, 1):
        assert torch.equal(pg.read([c], [0], [21])[0][0], x)
