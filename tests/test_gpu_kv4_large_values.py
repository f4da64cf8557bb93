"""Values that are very large or very small: sums of weights times values neither overflow nor vanish.

Weights before the division are up to 2^12, and 3000 tokens of values up to 4 * 2^93 sum to less than 2^12 * 2^12 * 2^95 = 2^119; the
smallest values, 2^-60 and less, are compared to the same relative bounds, for their products with weights above 2^-40 are normal
numbers and all weights below that together are off by 2^-40 of the largest value at most."""
import pytest
import torch

from tests.test_gpu_kv4 import make_cache, shape_of
from tests.test_gpu_kv4_many import definition, rows_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [90, 93, -60])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,before,rows", [((8, 2, 64), 3000, 9), ((32, 8, 128), 500, 17), ((64, 8, 128), 2000, 256), ((32, 8, 64), 2900, 100)])
def test_large_and_small_values(heads, before, rows, dtype, power):
    print("case", heads, before, rows, dtype, power, flush=True)
    nq, nkv, dim = heads
    kv = make_cache(shape_of(*heads, dtype), 1, before + rows)
    for n, seed in ((before, 1), (rows, 3)):
        kv.extend([0], [n])
        kv.append(0, rows_of(n, nkv, dim, dtype, seed), torch.ldexp(rows_of(n, nkv, dim, dtype, seed + 1).float().clamp(-4, 4), torch.tensor(power)).to(kv.dtype))
    q = rows_of(rows, nq, dim, dtype, 5)
    out = kv.attend(0, q)
    k, v = kv.read([0], [0], [before + rows])
    o, s, a, _, _ = definition(q, k[0], v[0], torch.arange(before + 1, before + rows + 1, device="cuda"))
    bound = ((2.0 ** -17 if dtype == "f32" else 2.0 ** -8) + 2.0 ** -18 * a) * s + 2.0 ** -100
    assert bool(((out.double() - o).abs() <= bound).all())
