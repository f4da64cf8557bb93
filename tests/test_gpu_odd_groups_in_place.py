"""Results over the queries where 3, 5 or 6 query heads share a head of the cache: the columns that a row's heads leave over read nothing that
another workgroup may have written already, so the results have the bits of those that lie elsewhere."""
import random

import pytest
import torch

from tests import test_gpu_kv4, test_gpu_pages
from tests.test_gpu_pages import fill, random_rows, random_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [(24, 8, 128), (40, 8, 64), (48, 8, 128)])
@pytest.mark.parametrize("cache", ["pages", "kv4"])
def test_bits_of_results_over_the_queries(cache, heads, dtype):
    nq, nkv, dim = heads
    r = random.Random(nq)
    rows = [r.choice([1, 2, 5, 6, 7, 11, 23]) for _ in range(40)]
    before = [r.randint(0, 900) for _ in rows]
    ours = test_gpu_pages if cache == "pages" else test_gpu_kv4
    shape = ours.shape_of(nq, nkv, dim, dtype)
    if cache == "pages":
        c = ours.make_cache(shape, len(rows), sum((b + n + 15) // 16 for b, n in zip(before, rows)))
    else:
        c = ours.make_cache(shape, len(rows), sum(before) + sum(rows) + 16 * len(rows))
    k, v = (random_rows(1000, nkv, dim, dtype, j) for j in (1, 2))
    for i, b in enumerate(before):
        fill(c, 0, i, k, v, b, 1000)
    n = sum(rows)
    if cache == "pages":
        c.extend(range(len(rows)), rows, [p for m in rows for p in random_tree(m, m)])
    else:
        c.extend(range(len(rows)), rows)
    c.append(0, k[:n].cuda(), v[:n].cuda())
    q = random_rows(n, nq, dim, dtype, 3).cuda()
    want = c.attend(0, q)
    for _ in range(5):
        x = q.clone()
        assert c.attend(0, x, out=x) is x
        assert torch.equal(x, want)
