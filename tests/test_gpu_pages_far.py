"""The paged cache where numbers get large: blocks beyond 4 GB of a pool, layers behind them, contexts of hundreds of thousands of tokens, passes larger
than what creation provides for (also while calls are recorded), other streams."""
import pytest
import torch

from paper_2605_13319_amd import nav
from tests.test_gpu_pages import attend_case, check_rows, fill, make_cache, random_rows, random_tree, reference, sees, shape_of

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_beyond_4_gb(dtype):
    nq, nkv, dim, n, rows = 16, 8, 128, 300, 12
    blocks = 80000  # 2.6 GB (bf16) of keys of a layer: 5.2 GB to its values' end, 10.5 to the second layer's
    pg = nav.PageCache(shape_of(nq, nkv, dim, dtype, layers=2), 4, blocks)
    pg.extend([0], [16 * (blocks - 60)])  # (takes the blocks in front)
    for layer in (0, 1):
        k, v = (random_rows(n + rows, nkv, dim, dtype, 10 * layer + j) for j in (1, 2))
        q = random_rows(rows, nq, dim, dtype, 10 * layer + 3)
        tree = random_tree(rows, 5)
        pg.truncate([1], [0])
        fill(pg, layer, 1, k, v, n)
        pg.extend([1], [rows], tree)
        pg.append(layer, k[n:].cuda(), v[n:].cuda())
        check_rows(pg.attend(layer, q.cuda()), *reference(q, k, v, sees(n, tree)), dtype)
        pg.copy([1], [2])
        pg.compact([2], [5], [[1, 2, 40]])
        at = [0, 1, 2, 3, 4, 6, 7, 45]
        for got, want in zip(pg.read([2], [0], [8], layer0=layer, n_layers=1), (k, v)):
            assert torch.equal(got[0].cpu(), want[at])


@gpu
def test_a_context_of_400000_tokens():
    nq, nkv, dim, n, rows = 4, 1, 64, 400000, 9
    pg = nav.PageCache(shape_of(nq, nkv, dim), 2, 26000)
    k, v = (random_rows(n + rows, nkv, dim, "bf16", j) for j in (1, 2))
    fill(pg, 0, 0, k, v, n, chunk=100000)
    pg.fork([0], [1], [n - 7])
    tree = random_tree(rows, 5)
    q = random_rows(2 * rows, nq, dim, "bf16", 3)
    pg.extend([0, 1], [rows, rows], tree * 2)
    pg.append(0, torch.cat([k[n:]] * 2).cuda(), torch.cat([v[n:]] * 2).cuda())
    out = pg.attend(0, q.cuda())
    check_rows(out[:rows], *reference(q[:rows], k, v, sees(n, tree)), "bf16")
    near = lambda x: torch.cat([x[:n - 7], x[n:]])
    check_rows(out[rows:], *reference(q[rows:], near(k), near(v), sees(n - 7, tree)), "bf16")


@gpu
def test_passes_larger_than_provided_for():
    """A recorded layer goes on working after a larger pass has made the scratch grow."""
    nq, nkv, dim, before, rows = 32, 1, 128, 3000, 20
    pg = make_cache(shape_of(nq, nkv, dim), 20, 700)
    k, v = (random_rows(before + rows, nkv, dim, "bf16", j) for j in (1, 2))
    q = random_rows(rows, nq, dim, "bf16", 3).cuda()
    tree = random_tree(rows, 4)
    fill(pg, 0, 0, k, v, before)
    pg.extend([0], [rows], tree)
    pg.append(0, k[before:].cuda(), v[before:].cuda())
    want = reference(q.cpu(), k, v, sees(before, tree))
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pg.attend(0, q, out=out)
    seqs, many = list(range(1, 19)), 200
    big_k, big_v = (random_rows(18 * many, nkv, dim, "bf16", j) for j in (5, 6))
    big_q = random_rows(18 * many, nq, dim, "bf16", 7)
    pg.extend(seqs, [many] * 18, random_tree(many, 8) * 18)
    pg.append(0, big_k.cuda(), big_v.cuda())
    got = pg.attend(0, big_q.cuda())
    for c in (0, 17):
        part = slice(c * many, (c + 1) * many)
        check_rows(got[part], *reference(big_q[part], big_k[part], big_v[part], sees(0, random_tree(many, 8))), "bf16")
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check_rows(out, *want, "bf16")


@gpu
def test_passes_on_another_stream():
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        pg, q, out = attend_case(8, 2, 128, "bf16", [300, 40], [17, 9], [random_tree(17, 1), random_tree(9, 2)])
        pg.fork([0], [1], [60])
        pg.compact([1], [3], [[5, 6, 50]])
        text = [x.cpu() for x in pg.read([0], [0], [60])]
        for got, was in zip(pg.read([1], [0], [6]), text):
            assert torch.equal(got.cpu().view(torch.int16), was[:, [0, 1, 2, 8, 9, 53]].view(torch.int16))  # (layer 0 holds the pool's NaN)
        side.synchronize()


@gpu
def test_a_pass_allocates_nothing_on_the_device():
    pg = make_cache(shape_of(32, 8, 128), 16, 2000)
    k = random_rows(16 * 64, 8, 128, "bf16", 1).cuda()
    q = random_rows(16 * 64, 32, 128, "bf16", 2).cuda()
    out = torch.empty_like(q)
    fill(pg, 0, 0, k[:1000], k[:1000], 1000)
    pg.fork([0] * 15, list(range(1, 16)))
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    pg.extend(list(range(16)), [64] * 16, random_tree(64, 3) * 16)
    pg.append(0, k, k)
    pg.attend(0, q, out=out)
    pg.compact(list(range(16)), [1000] * 16, [[0, 1, 5]] * 16)
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free


@gpu
def test_one_long_context_among_many_rows():
    """Only its rows have splits to join."""
    nq, nkv, dim, n, rows, clients = 128, 1, 64, 40000, 700, 12
    pg = nav.PageCache(shape_of(nq, nkv, dim), 1 + clients, n // 16 + 2 + clients * 45)
    k, v = (random_rows(n + 1, nkv, dim, "bf16", j) for j in (1, 2))
    fill(pg, 0, 5, k, v, n, chunk=20000)
    ks, vs = (random_rows(rows, nkv, dim, "bf16", j) for j in (3, 4))
    q = random_rows(1 + clients * rows, nq, dim, "bf16", 5)
    others = [c for c in range(1 + clients) if c != 5]
    pg.extend(others[:7] + [5] + others[7:], [rows] * 7 + [1] + [rows] * (clients - 7))
    at = 7 * rows
    put = lambda one, x: torch.cat([x] * 7 + [one[n:]] + [x] * (clients - 7)).cuda()
    pg.append(0, put(k, ks), put(v, vs))
    out = pg.attend(0, q.cuda())
    check_rows(out[at:at + 1], *reference(q[at:at + 1], k, v, sees(n, [-1])), "bf16")
    for first in (0, at + 1):
        part = slice(first, first + rows)
        check_rows(out[part], *reference(q[part], ks, vs, sees(0, list(range(-1, rows - 1)))), "bf16")
