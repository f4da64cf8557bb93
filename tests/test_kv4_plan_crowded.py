"""Passes of so many clients that the device is filled several times over: a long context among them is cut all the same, for its last
split is what the pass waits for; contexts that are alike are not.  The plan on the host, and such a pass against its definition."""
import pytest
import torch

from paper_2605_13319_amd import nav
from tests.test_gpu_kv4 import check_rows, shape_of
from tests.test_gpu_kv4_many import definition, rows_of
from tests.test_kv4_plan import kinds, plan  # noqa: F401 (a fixture)


@pytest.mark.parametrize("last", [False, True])
@pytest.mark.parametrize("heads,n,rows", [((40, 40, 128), 52, 1), ((40, 40, 128), 64, 1), ((32, 8, 128), 256, 1), ((32, 8, 128), 90, 9),
                                          ((32, 8, 64), 256, 4), ((128, 16, 64), 200, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_long_context_among_short_ones_is_cut(plan, heads, n, rows, last, dtype):  # noqa: F811
    before = [300] * n
    before[-1 if last else 0] = 131072
    got = kinds(plan, heads, dtype, before, [rows] * n)
    # (32 tokens of a tile take 0.08 us and more: 16 splits of 8192 tokens 20, uncut 330)
    assert got[-1 if last else 0][1] >= 16
    assert all(s == 1 for _, s in (got[:-1] if last else got[1:]))


@pytest.mark.parametrize("length", [300, 4096, 30000])
@pytest.mark.parametrize("heads,n", [((40, 40, 128), 64), ((32, 8, 128), 256), ((128, 16, 64), 200)])
def test_contexts_that_are_alike_are_not(plan, heads, n, length):  # noqa: F811
    assert {s for _, s in kinds(plan, heads, "bf16", [length] * n, [1] * n)} == {1}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nkv,dim", [(40, 40, 128), (16, 16, 64)])
def test_against_the_definition(nq, nkv, dim, dtype):
    n, long = 150, 30000
    before = [(c * 37) % 100 for c in range(n)]
    before[70] = long
    kv = nav.KV4Cache(shape_of(nq, nkv, dim, dtype), n, 8 * n + long // 16 + 8)
    kv.pool.fill_(255)
    ids = [c for c in range(n) if before[c]]
    kv.extend(ids, [before[c] for c in ids])
    kv.append(0, rows_of(sum(before), nkv, dim, dtype, 1), rows_of(sum(before), nkv, dim, dtype, 2))
    kv.extend(list(range(n)), [1] * n)
    kv.append(0, rows_of(n, nkv, dim, dtype, 3), rows_of(n, nkv, dim, dtype, 4))
    q = rows_of(n, nq, dim, dtype, 5)
    mass = torch.full((n, 1, nkv, long + 1), torch.nan, device="cuda")
    out = kv.attend(0, q, mass=mass, decay=0.0)
    for c in range(n):
        k, v = kv.read([c], [0], [before[c] + 1])
        o, s, a, w, big = definition(q[c:c + 1], k[0], v[0], torch.tensor([before[c] + 1], device="cuda"))
        check_rows(out[c:c + 1], o.cpu(), s.cpu(), a.cpu(), dtype)
        assert bool(((mass[c, 0, :, :before[c] + 1].double() - w).abs() <= 2.0 ** -18 * (1 + big[:, None]) * w + 1e-30).all())
