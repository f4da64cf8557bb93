"""Values that are very large or very small: sums of weights times values neither overflow nor vanish.

Weights before the division are up to 2^8, and 4096 tokens of values up to 2^100 sum to at most 2^12 * 2^8 * 2^100 = 2^120; the smallest
values, 2^-60 and less, are compared to the same relative bounds, for their products with weights above 2^-40 are normal numbers and all
weights below that together are off by 2^-40 * 2^12 of the largest value at most.  Bounds as in test_gpu_pages.py."""
import pytest
import torch

from tests.test_gpu_pages import check_rows, fill, make_cache, random_rows, random_tree, reference, sees, shape_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [98, -60])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,before,rows", [((8, 2, 64), 3000, 9), ((8, 2, 128), 500, 33), ((32, 8, 128), 2000, 200), ((16, 4, 64), 2900, 100)])
def test_large_and_small_values(heads, before, rows, dtype, power):
    nq, nkv, dim = heads
    pg = make_cache(shape_of(*heads, dtype), 1, (before + rows + 15) // 16)
    k, v = (random_rows(before + rows, nkv, dim, dtype, j) for j in (1, 2))
    v = torch.ldexp(v.float().clamp(-4, 4), torch.tensor(power)).to(v.dtype)
    fill(pg, 0, 0, k, v, before)
    tree = random_tree(rows, 3)
    pg.extend([0], [rows], tree)
    pg.append(0, k[before:].cuda(), v[before:].cuda())
    q = random_rows(rows, nq, dim, dtype, 5)
    check_rows(pg.attend(0, q.cuda()), *reference(q, k, v, sees(before, tree)), dtype)
