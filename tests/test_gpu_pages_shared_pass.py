"""Clients that share the rows of a pass that has not ended: what the other client holds stays as it was when it became a copy."""
import pytest
import torch

from paper_2605_13319_amd import nav
from tests.test_gpu_pages import make_cache, random_rows, shape_of

gpu = pytest.mark.gpu
NKV, DIM = 2, 64


def rows(n, seed):
    return random_rows(n, NKV, DIM, "bf16", seed).cuda()


def refused(pg, layer, x):
    with pytest.raises(nav.PipesdError) as e:
        pg.append(layer, x, x)
    assert e.value.status == nav.ESTATE


@gpu
@pytest.mark.parametrize("before", [0, 16, 21])
def test_rows_that_another_client_holds_as_well_are_not_written(before):
    pg = make_cache(shape_of(4, NKV, DIM, layers=2), 4, 40)
    if before:
        pg.extend([0], [before])
        for layer in (0, 1):
            pg.append(layer, rows(before, 1), rows(before, 1))
    pg.extend([0, 1], [20, 3])
    for layer in (0, 1):
        pg.append(layer, rows(23, 2), rows(23, 3))
    pg.fork([0], [2], [before + 5])
    held = [x.clone() for x in pg.read([2], [0], [before + 5])]
    refused(pg, 0, rows(23, 4))
    refused(pg, 1, rows(23, 4))
    for got, was in zip(pg.read([2], [0], [before + 5]), held):
        assert torch.equal(got, was)
    q = random_rows(23, 4, DIM, "bf16", 5).cuda()
    pg.attend(0, q)  # (the pass goes on reading)
    pg.fork([2], [3])  # (a copy's copy)
    refused(pg, 0, rows(23, 4))
    pg.truncate([2, 3], [0, 0])
    refused(pg, 0, rows(23, 4))  # (for this pass it stays so)
    pg.extend([0, 1], [1, 1])
    pg.append(0, rows(2, 6), rows(2, 6))


@gpu
def test_what_does_not_share_a_pass_does_not_stop_it():
    pg = make_cache(shape_of(4, NKV, DIM, layers=2), 5, 60)
    pg.extend([0, 1], [21, 30])
    for layer in (0, 1):
        pg.append(layer, rows(51, 1), rows(51, 1))
    pg.extend([0], [20])
    x = rows(20, 2)
    pg.append(0, x, x)
    pg.fork([0, 1, 1], [2, 3, 4], [21, 30, 7])  # the text before the pass; clients that are not in it
    pg.copy([0], [4])  # has blocks of its own, and of this pass what has been appended
    y = rows(20, 3)
    pg.append(0, y, y)
    pg.append(1, y, y)
    assert torch.equal(pg.read([0], [21], [20])[0], torch.stack([y, y]))
    assert torch.equal(pg.read([4], [21], [20], 0, 1)[0][0], x)
    for c, n in ((0, 21), (2, 21)):
        assert torch.equal(pg.read([c], [0], [n])[0], torch.stack([rows(51, 1)[:21]] * 2))
    pg.extend([2, 0], [2, 2])  # (the shared block, which both write into, is one's own for each)
    z = rows(4, 4)
    pg.append(0, z, z)
    assert torch.equal(pg.read([2], [20], [3], 0, 1)[0][0], torch.cat([rows(51, 1)[20:21], z[:2]]))
    assert torch.equal(pg.read([0], [21], [22], 0, 1)[0][0], torch.cat([y, z[2:]]))
