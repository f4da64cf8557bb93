"""Results of attention written where its queries are: the same result as elsewhere where no weights are asked for, and refused
where it cannot be right (the weights are formed from the queries again, and rows of partly overlapping buffers are read
after others have been written).  Columns of one wider matrix do not overlap."""
import ctypes as C

import pytest
import torch

from paper_2605_13319_amd import nav
from tests.test_gpu_kv4 import host_cache, make_cache, random_rows, refused, shape_of

gpu = pytest.mark.gpu


def filled(heads, dtype, before, rows):
    nq, nkv, dim = heads
    kv = make_cache(shape_of(*heads, dtype), 1, before + rows)
    for n, seed in ((before, 1), (rows, 3)):
        kv.extend([0], [n])
        kv.append(0, random_rows(n, nkv, dim, dtype, seed).cuda(), random_rows(n, nkv, dim, dtype, seed + 1).cuda())
    return kv, random_rows(rows, nq, dim, dtype, 5).cuda()


CASES = [((8, 2, 64), "bf16", 100, 9), ((6, 2, 128), "f32", 3000, 17), ((7, 1, 128), "bf16", 7003, 1024)]  # (the last: eight tiles a workgroup)


@gpu
@pytest.mark.parametrize("heads,dtype,before,rows", CASES)
def test_in_place_of_the_queries(heads, dtype, before, rows):
    kv, q = filled(heads, dtype, before, rows)
    want, x = kv.attend(0, q), q.clone()
    assert kv.attend(0, x, out=x) is x
    assert torch.equal(x, want)


@gpu
@pytest.mark.parametrize("heads,dtype,before,rows", CASES)
def test_in_place_with_weights_is_refused(heads, dtype, before, rows):
    kv, q = filled(heads, dtype, before, rows)
    was = q.clone()
    mass = torch.full((1, 1, heads[1], before + rows), 5.0, device="cuda")
    refused(nav.EINVAL, lambda: kv.attend(0, q, out=q, mass=mass))
    assert torch.equal(q, was) and bool((mass == 5.0).all())
    kv.attend(0, q, mass=mass)  # (the pass goes on)


@gpu
def test_columns_of_one_matrix_and_rows_that_overlap():
    (nq, nkv, dim), n = (4, 2, 64), 5
    kv, q = filled((nq, nkv, dim), "bf16", 20, n)
    want = kv.attend(0, q)
    mass = torch.zeros(1, 1, nkv, 25, device="cuda")
    other = torch.zeros_like(mass)
    kv.attend(0, q, mass=other, decay=0.0)
    wide = torch.zeros(n, 3 * nq * dim, dtype=torch.bfloat16, device="cuda")
    for a, b in ((0, 1), (1, 0), (2, 0), (1, 2)):  # queries and results side by side, in either order
        wide.zero_()
        wide[:, a * 256:a * 256 + 256] = q.flatten(1)
        kv.attend(0, wide[:, a * 256:a * 256 + 256], out=wide[:, b * 256:b * 256 + 256], mass=mass, decay=0.0)
        assert torch.equal(wide[:, b * 256:b * 256 + 256].view_as(want), want) and torch.equal(mass, other)
    long = torch.zeros(2 * n, nq, dim, dtype=torch.bfloat16, device="cuda")  # rows in turn
    long[::2] = q
    kv.attend(0, long[::2], out=long[1::2], mass=mass, decay=0.0)
    assert torch.equal(long[1::2], want) and torch.equal(long[::2], q)
    for weights in (None, mass):
        refused(nav.EINVAL, lambda: kv.attend(0, wide[:, :256], out=wide[:, 8:264], mass=weights))
        refused(nav.EINVAL, lambda: kv.attend(0, long[:n], out=long[1:n + 1], mass=weights))
        refused(nav.EINVAL, lambda: kv.attend(0, long[::2], out=long[4:4 + n], mass=weights))


def test_overlaps_on_the_host():
    """(the check comes after the arguments' and before any device work)"""
    lib, kv = nav._lib, host_cache()
    kv.extend([0], [3])
    p = 1 << 20

    def at(o, qs=256, os_=256, m=None):
        return lib.pipesd_kv4_attend(kv.handle, 0, p, qs, None, o, os_, m, 64, 1.0, None)
    row = 256 * 2
    good = [at(p), at(p + 3 * row), at(p - 3 * row), at(p + row, 512, 512), at(p + row, 512, 1024), at(p + 5 * row, 512, 256, C.c_void_p(4096))]
    bad = [at(p, m=C.c_void_p(4096)), at(p, 256, 512), at(p + 16), at(p - 16), at(p + 2 * row), at(p - 2 * row), at(p + row + 16, 512, 512),
           at(p + 2 * row, 512, 256), at(p + 3 * row, 512, 256), at(p + row - 16, 512, 256), at(p + 4 * row - 32, 512, 512)]
    assert set(good) == {nav.ESTATE}  # (no pool)
    assert set(bad) == {nav.EINVAL}


def test_overlaps_of_all_strides_on_the_host():
    """Against every row with every other."""
    import random
    lib, r = nav._lib, random.Random(3)
    seen = {nav.EINVAL: 0, nav.ESTATE: 0}
    for rows in (1, 2, 3, 7):
        kv = nav.KV4Cache(shape_of(1, 1, 64, "f32"), 1, 8, on_device=False)
        kv.extend([0], [rows])
        for _ in range(1500):
            p, width = 1 << 20, 64 * 4
            qs = 64 + 4 * r.randrange(40)
            os_ = r.choice([qs, 64 + 4 * r.randrange(40)])
            o = p + 16 * r.randrange(-120, 121)
            shared = any(p + i * qs * 4 < o + j * os_ * 4 + width and o + j * os_ * 4 < p + i * qs * 4 + width for i in range(rows) for j in range(rows))
            for mass in (None, C.c_void_p(4096)):
                want = nav.EINVAL if shared and not (mass is None and o == p and os_ == qs) else nav.ESTATE
                assert lib.pipesd_kv4_attend(kv.handle, 0, p, qs, None, o, os_, mass, 64, 1.0, None) == want, (rows, qs, os_, o - p, mass)
                seen[want] += 1
    assert min(seen.values()) > 1000
