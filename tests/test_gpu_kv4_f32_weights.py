"""Weights of an fp32 model's attention over the 4-bit cache have 24 bits, as fp32 numbers have.

A row sees five tokens; only one of them has values, and not the one with the most weight, so a result is that token's weight times an
exact number.  Scores come from one channel (a query's fp32 number, exactly in three pieces, times 1, 1.5 or 2), and differ by
at most 1 in base 2.

Bound, in units of 2^-23 of the result, set before the first run: the constant log2(e) / sqrt(d) is off by 1 relative to differences of at
most 1: 0.7; the score's own rounding and the sum with the maximum, numbers below 4: 0.7 each and once more for the maximum of
another wave: 2.1; two exponentials, 1 each: 2; four sums of weights and a product with a wave's factor, 0.5 each: 2.5, as much again
for the values' products; 1 / l and its product: 1.  10.8, below 2^-23 * 16 = 2^-19.  Weights cut to 16 bits are off by up to 2^-18."""
import math

import pytest
import torch

from tests.test_gpu_kv4 import make_cache, shape_of

pytestmark = pytest.mark.gpu

TOKENS = 5


def error(heads, dtype, before, rows, heavy, seen, seed):
    """The largest relative error of the results."""
    nq, nkv, dim = heads
    kv = make_cache(shape_of(*heads, dtype), 1, before + rows)
    g = torch.Generator().manual_seed(seed)
    k, v = torch.zeros(2, before + rows, nkv, dim)
    grid = torch.tensor([1.0, 1.5, 1.0, 1.5, 1.0])
    k[:TOKENS, :, 3] = grid[:, None]
    k[heavy, :, 3] = 2.0
    v[seen] = torch.tensor([1.0, -2.0, 3.0, 6.0]).repeat(dim // 4)
    v[TOKENS:] = 5.0  # (hidden)
    type_ = torch.float32 if dtype == "f32" else torch.bfloat16
    k, v = k.to(type_).cuda(), v.to(type_).cuda()
    for first, n in ((0, before), (before, rows)):
        kv.extend([0], [n])
        kv.append(0, k[first:first + n], v[first:first + n])
    q = torch.zeros(rows, nq, dim)
    # scores q k / sqrt(dim) with k from 1 to 2 that differ by at most 1 in base 2
    q[..., 3] = torch.rand(rows, nq, generator=g) * math.log(2) * math.sqrt(dim)
    q = q.to(type_).cuda()
    out = kv.attend(0, q, limits=torch.full((rows,), TOKENS, dtype=torch.int32, device="cuda"))
    z = q[..., 3:4].double() * k[:TOKENS, 0, 3].double() / math.sqrt(dim)
    want = z.softmax(-1)[..., seen:seen + 1] * v[seen, 0].double()
    return float(((out.double() - want).abs() / want.abs()).max())


@pytest.mark.parametrize("heavy,seen", [(0, 1), (4, 0), (2, 3)])
@pytest.mark.parametrize("heads,before,rows", [
    ((4, 4, 64), 100, 40),         # one tile a workgroup, one split
    ((32, 8, 128), 3000, 17),      # several splits
    ((32, 32, 64), 15000, 512),    # eight tiles a workgroup
    ((32, 4, 128), 9000, 1024),
])
def test_results_are_as_good_as_fp32(heads, before, rows, heavy, seen):
    print("case", heads, before, rows, heavy, seen, flush=True)
    assert error(heads, "f32", before, rows, heavy, seen, 10 * heavy + seen) <= 2.0 ** -19
