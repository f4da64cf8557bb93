"""Clients that are in a pass without new rows: their weights are decayed as everyone's are, and nothing else of them changes.

What is compared: an idle client's weight is the fp32 product of the decay and what the buffer held, so exactly that; with decay 0
it is 0 whatever the buffer held, with decay 1 what it was.  Weights beyond a client's length, of other layers, and of clients that
are not in the pass stay."""
import pytest
import torch

from tests.test_gpu_kv4 import make_cache, random_rows, refused, shape_of
from paper_2605_13319_amd import nav

pytestmark = pytest.mark.gpu


def filled(before, layers=2, nq=4, nkv=2, dim=64, dtype="bf16", spare=40):
    kv = make_cache(shape_of(nq, nkv, dim, dtype, layers), len(before), max(before) + spare)
    for c, n in enumerate(before):
        for f in range(0, n, 20000):
            m = min(20000, n - f)
            kv.extend([c], [m])
            x = random_rows(m, nkv, dim, dtype, c).cuda()
            for layer in range(layers):
                kv.append(layer, x, x)
    return kv


def attended(kv, ids, rows, weights, decay, layer=1):
    s = kv.shape
    dtype = "bf16" if kv.dtype == torch.bfloat16 else "f32"
    kv.extend(ids, rows)
    n = sum(rows)
    x = random_rows(n, s.n_kv_heads, s.head_dim, dtype, 7).cuda()
    kv.append(layer, x, x)
    mass = weights.cuda()
    kv.attend(layer, random_rows(n, s.n_q_heads, s.head_dim, dtype, 8).cuda(), mass=mass, decay=decay)
    return mass.cpu()


def check_idle(kv, before, ids, rows, weights, mass, decay, layer=1):
    for c, n in enumerate(before):
        busy = c in ids and rows[ids.index(c)] > 0
        want = weights[c].clone()
        if c in ids and not busy:
            want[layer, :, :n] = 0.0 if decay == 0 else want[layer, :, :n] * torch.tensor(decay, dtype=torch.float32)
        if busy:
            end = n + rows[ids.index(c)]
            assert not torch.isnan(mass[c, layer, :, :end]).any()
            want[layer, :, :end] = mass[c, layer, :, :end]
        assert torch.equal(mass[c].view(torch.int32), want.view(torch.int32)), c


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("decay", [0.0, 0.75, 0.9, 1.0])
def test_idle_clients_of_a_pass_are_decayed(decay, dtype):
    before, ids, rows = [0, 1, 130, 1023, 1024, 2050, 33], [5, 3, 0, 2, 1, 4], [3, 0, 0, 0, 0, 1]
    kv = filled(before, dtype=dtype)
    w = torch.rand(len(before), 2, 2, 2101, generator=torch.Generator().manual_seed(3)).float()
    if decay == 0:
        w[:, 1, :, ::3] = torch.nan
        w[:, 1, :, 1::7] = torch.inf
    check_idle(kv, before, ids, rows, w, attended(kv, ids, rows, w, decay), decay)


def test_more_idle_clients_than_a_launch_takes():
    before = [(29 * c) % 97 for c in range(70)]
    ids = list(range(69, -1, -1))
    rows = [1 if c == 11 else 0 for c in ids]
    kv = filled(before)
    w = torch.rand(70, 2, 2, 140, generator=torch.Generator().manual_seed(4)).float()
    check_idle(kv, before, ids, rows, w, attended(kv, ids, rows, w, 0.5), 0.5)


def test_a_long_idle_client():
    before, ids, rows = [70001, 5], [0, 1], [0, 2]
    kv = filled(before, layers=2)
    w = torch.rand(2, 2, 2, 70050, generator=torch.Generator().manual_seed(5)).float()
    check_idle(kv, before, ids, rows, w, attended(kv, ids, rows, w, 0.3), 0.3)


def test_a_cut_goes_by_weights_that_were_cleared():
    """An idle client's weights of an earlier text are gone with decay 0: a cut then keeps the lowest indices."""
    kv = filled([50, 3], layers=1)
    w = torch.full((2, 1, 2, 60), torch.nan)
    w[0, 0, :, 20:45] = 9.0
    mass = attended(kv, [0, 1], [0, 1], w, 0.0, layer=0).cuda()
    kept = kv.evict([0], [0], 10, 2, mass)
    assert kept[0, 0].tolist() == [[0, 1, 2, 3, 4, 5, 6, 7, 48, 49]] * 2


def test_an_idle_client_longer_than_its_weights_is_refused():
    kv = filled([64, 3], layers=1)
    kv.extend([0, 1], [0, 1])
    x, q = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    kv.append(0, x, x)
    for decay in (0.0, 0.5, 1.0):
        refused(nav.EINVAL, lambda: kv.attend(0, q, mass=torch.zeros(2, 1, 2, 63, device="cuda"), decay=decay))
    kv.attend(0, q, mass=torch.zeros(2, 1, 2, 64, device="cuda"))
