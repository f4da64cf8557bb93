"""The weights' buffer is the caller's: what it holds for tokens of a pass that asked for no weights counts in the next that does, also
where it is what a forgotten or cut token left; cleared before, as the interface asks, such a token starts at 0."""
import pytest
import torch

from tests.test_gpu_kv4 import make_cache, random_rows, shape_of

pytestmark = pytest.mark.gpu

NQ, NKV, DIM = 4, 2, 64


def rows(n, seed, heads=NKV):
    return random_rows(n, heads, DIM, "bf16", seed).cuda()


@pytest.mark.parametrize("clear", [False, True])
@pytest.mark.parametrize("how", ["truncate", "evict"])
def test_weights_of_tokens_that_came_in_a_pass_without(how, clear):
    kv = make_cache(shape_of(NQ, NKV, DIM), 1, 200)
    mass = torch.full((1, 1, NKV, 150), torch.nan, device="cuda")
    kv.extend([0], [100])
    kv.append(0, rows(100, 1), rows(100, 2))
    kv.attend(0, rows(100, 3, NQ), mass=mass, decay=0.0)
    if how == "truncate":
        kv.truncate([0], [60])
    else:
        kv.evict([0], [0], 60, 10, mass)
    left = mass.clone()
    if clear:
        mass[..., 60:] = 0.0
    kv.extend([0], [20])  # asks for no weights
    kv.append(0, rows(20, 4), rows(20, 5))
    kv.attend(0, rows(20, 6, NQ))
    assert torch.equal(mass[..., :60], left[..., :60])
    kv.extend([0], [3])
    kv.append(0, rows(3, 7), rows(3, 8))
    q = rows(3, 9, NQ)
    given = torch.zeros_like(mass)
    kv.attend(0, q, mass=given, decay=0.0)
    kv.attend(0, q, mass=mass, decay=0.5)
    old = 0.5 * left
    if clear:
        old[..., 60:] = 0.0
    old[..., 80:] = 0.0  # (the pass's own)
    assert torch.equal(mass[..., :83], (old + given)[..., :83])
    assert bool((mass[..., 60:80] > given[..., 60:80]).any()) != clear
