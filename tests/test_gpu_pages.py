"""The paged cache of operators against its definition in 64 bits: rows in and out, attention of chains and trees (both dtypes and head
sizes, few and many rows, short and long contexts, ragged clients, strides), values that are no numbers where rows do not see
them, clients that share blocks, compaction, recorded passes.  The pool starts as bytes of ones, so whatever is read beyond a
client's tokens is not a number.

Bounds, set before the first run.  A row o = sum p v, with S = sum p |v| and A = the largest sum |q k| / sqrt(d) of its row:
 * scores: 128 products (exact in fp32 for bf16 numbers, rounded for fp32 ones), summed in fp32 in some order: rounding errors of 2^-24
   that add like a random walk over 256 operations are 2^-20 of sum |q k|, four times that allowed; an error of a score is the
   relative error of its weight: 2^-18 A;
 * bf16: results are rounded to 8 bits, half a step is 2^-8 |o| <= 2^-8 S; weights are cut to 16 bits, 2^-17 S;
 * fp32: weights are fp32; exponentials and sums over up to 2^13 steps that add like a random walk: 2^-24 * 2^6.5, 2^-17 S allowed.
Rows that are stored, moved and copied are compared exactly."""
import math
import random

import pytest
import torch

from paper_2605_13319_amd import inputs as I
from paper_2605_13319_amd import nav

gpu = pytest.mark.gpu


def shape_of(nq, nkv, dim, dtype="bf16", layers=1):
    return I.ModelShape("pages", layers, 512, nq, nkv, dim, 512, 512, dtype=I.DTYPE_F32 if dtype == "f32" else I.DTYPE_BF16)


def make_cache(shape, max_seqs, blocks):
    pg = nav.PageCache(shape, max_seqs, blocks)
    pg.pool.fill_(255)
    return pg


def random_rows(rows, heads, dim, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, heads, dim, generator=g) * scale
    x = x * (1 + 3 * (torch.rand(heads, dim, generator=g) < 0.05))
    return x.to(torch.float32 if dtype == "f32" else torch.bfloat16)


def random_tree(rows, seed, roots=False):
    r = random.Random(seed)
    return [-1] + [r.randint(-1 if roots else 0, i - 1) if r.random() < 0.5 else i - 1 for i in range(1, rows)]


def sees(before, parents):
    m = torch.zeros(len(parents), before + len(parents), dtype=torch.bool)
    m[:, :before] = True
    for i, p in enumerate(parents):
        if p >= 0:
            m[i] |= m[p]
        m[i, before + i] = True
    return m


def reference(q, k, v, seen):
    """(o, S, A) of one client, in 64 bits; what a row does not see is left out, not multiplied by 0."""
    rows, nq, dim = q.shape
    nkv = k.shape[1]
    group = nq // nkv
    q, k, v = q.double(), k.double(), v.double()
    o, s, a = (torch.zeros(rows, nq, n, dtype=torch.float64) for n in (dim, dim, 1))
    whole = bool(torch.isfinite(k).all() and torch.isfinite(v).all())
    for h in range(nkv):
        heads = slice(h * group, (h + 1) * group)
        qh = q[:, heads].reshape(rows * group, dim)
        hidden = ~seen.repeat_interleave(group, 0)
        z = (qh @ k[:, h].T / math.sqrt(dim)).masked_fill(hidden, -torch.inf)
        big = (qh.abs() @ k[:, h].abs().T / math.sqrt(dim)).masked_fill(hidden, 0).amax(-1)
        w = torch.softmax(z, -1)
        if whole:
            oh, sh = w @ v[:, h], w @ v[:, h].abs()
        else:
            oh = torch.stack([x[~m] @ v[:, h][~m] for x, m in zip(w, hidden)])
            sh = torch.stack([x[~m] @ v[:, h][~m].abs() for x, m in zip(w, hidden)])
        o[:, heads], s[:, heads], a[:, heads] = oh.view(rows, group, dim), sh.view(rows, group, dim), big.view(rows, group, 1)
    return o, s, a


def check_rows(got, want, s, a, dtype):
    got = got.cpu().double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine)
    err = (got - want).abs()
    bound = ((2.0 ** -17 if dtype == "f32" else 2.0 ** -8 + 2.0 ** -17) + 2.0 ** -18 * a) * s + 2.0 ** -100
    worst = float((err - bound)[fine].max()) if fine.any() else 0.0
    assert worst <= 0, (worst, float(err[fine].max()))


def fill(pg, layer, c, k, v, n, chunk=700):
    for f in range(0, n, chunk):
        m = min(chunk, n - f)
        pg.extend([c], [m])
        pg.append(layer, k[f:f + m].cuda(), v[f:f + m].cuda())


# ---- rows in and out -----------------------------------------------------------------------------


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nkv,dim", [(1, 128), (8, 64), (5, 128)])
def test_ragged_passes_keep_every_client_apart(nkv, dim, dtype):
    shape = shape_of(nkv * 2, nkv, dim, dtype, layers=3)
    pg = make_cache(shape, 5, 40)
    want = {c: [[], []] for c in range(5)}
    for step, (ids, ns) in enumerate([([0, 1, 2], [1, 17, 40]), ([4, 2], [3, 1]), ([1, 0, 3, 4], [16, 0, 15, 29]), ([2], [50])]):
        n = sum(ns)
        pg.extend(ids, ns)
        parts = []
        for layer in range(3):
            k, v = (random_rows(n, nkv, dim, dtype, 100 * step + 10 * layer + j) for j in (0, 1))
            wide = torch.empty(n, 2 * nkv * dim + 16, dtype=k.dtype, device="cuda")  # rows of a wider matrix, as fused projections leave them
            wide[:, :nkv * dim], wide[:, nkv * dim + 16:] = k.flatten(1).cuda(), v.flatten(1).cuda()
            pg.append(layer, wide[:, :nkv * dim], wide[:, nkv * dim + 16:])
            parts.append((k, v))
        r = 0
        for c, m in zip(ids, ns):
            for j in (0, 1):
                want[c][j].append(torch.stack([p[j][r:r + m] for p in parts]))
            r += m
    ids = [3, 0, 2, 1, 4]
    lens = [pg.length(c) for c in ids]
    assert lens == [15, 1, 91, 33, 32]
    for j, got in enumerate(pg.read(ids, [0] * 5, lens)):
        assert torch.equal(got.cpu(), torch.cat([torch.cat(want[c][j], 1) for c in ids], 1))
    gk, _ = pg.read([2, 1], [13, 32], [30, 1], layer0=1, n_layers=1)
    assert torch.equal(gk.cpu(), torch.cat([torch.cat(want[2][0], 1)[1:2, 13:43], torch.cat(want[1][0], 1)[1:2, 32:33]], 1))
    assert pg.read([0], [1], [0])[0].shape == (3, 0, nkv, dim)


@gpu
@pytest.mark.parametrize("dtype,nkv,dim", [("bf16", 2, 64), ("bf16", 3, 128), ("f32", 2, 128), ("f32", 1, 64)])
def test_random_calls_leave_every_client_its_own_text(dtype, nkv, dim):
    """Clients are forked, copied, cut, compacted and go on by themselves: what each holds is what it should, whoever shares what."""
    r = random.Random(nkv * dim + (dtype == "f32"))
    clients, blocks, layers = 6, 60, 2
    pg = make_cache(shape_of(nkv, nkv, dim, dtype, layers), clients, blocks)
    text, made, big = [[] for _ in range(clients)], 0, 0
    store = [[], []]  # a row by its number: [layer][head][dim]
    for step in range(120):
        do = r.choice(["extend", "extend", "extend", "cut", "fork", "copy", "compact", "compact"])
        ids = r.sample(range(clients), r.randint(1, clients))
        try:
            if do == "extend":
                ns = [r.choice([0, 1, 1, 5, 16, 40, 70]) for _ in ids]
                n = sum(ns)
                if n == 0:
                    continue
                pg.extend(ids, ns)
                rows = [random_rows(n, layers * nkv, dim, dtype, 2 * step + j).view(n, layers, nkv, dim) for j in (0, 1)]
                for layer in range(layers):
                    pg.append(layer, rows[0][:, layer].contiguous().cuda(), rows[1][:, layer].contiguous().cuda())
                for j in (0, 1):
                    store[j].append(rows[j])
                for c, m in zip(ids, ns):
                    text[c] += range(made, made + m)
                    made += m
            elif do == "cut":
                ns = [r.randint(0, len(text[c])) for c in ids]
                pg.truncate(ids, ns)
                for c, n in zip(ids, ns):
                    del text[c][n:]
            elif do in ("fork", "copy"):
                into = ids[:r.randint(1, len(ids))]
                rest = [c for c in range(clients) if c not in into]
                if not rest:
                    continue
                src = [r.choice(rest) for _ in into]
                ns = [r.choice([len(text[c]), r.randint(0, len(text[c]))]) for c in src]
                getattr(pg, do)(src, into, ns)
                for c, t, n in zip(src, into, ns):
                    text[t] = text[c][:n]
            else:
                firsts = [r.choice([0, r.randint(0, len(text[c]))]) for c in ids]
                kept = [sorted(r.sample(range(len(text[c]) - f), r.randint(0, len(text[c]) - f))) for c, f in zip(ids, firsts)]
                pg.compact(ids, firsts, kept)
                big = max(big, sum(map(len, kept)))
                for c, f, k in zip(ids, firsts, kept):
                    text[c] = text[c][:f] + [text[c][f + j] for j in k]
        except nav.PipesdError as e:
            assert e.status == nav.ENOMEM
            free = [c for c in range(clients) if text[c]]
            c = r.choice(free)
            pg.truncate([c], [len(text[c]) // 3])
            del text[c][len(text[c]) // 3:]
        if step % 6 == 5:
            lens = [pg.length(c) for c in range(clients)]
            assert lens == [len(t) for t in text]
            at = torch.tensor([i for t in text for i in t], dtype=torch.int64)
            for j, got in enumerate(pg.read(range(clients), [0] * clients, lens)):
                if made:
                    assert torch.equal(got.cpu(), torch.cat(store[j])[at].transpose(0, 1)), (step, j)
    assert big > 100  # (of one call)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_compactions(dtype):
    """More tokens than a launch moves, over themselves; and behind a beginning that another client shares."""
    nkv, dim, n = 2, 128, 3000
    pg = make_cache(shape_of(nkv, nkv, dim, dtype), 3, 600)
    k, v = (random_rows(n, nkv, dim, dtype, j) for j in (1, 2))
    fill(pg, 0, 0, k, v, n)
    pg.fork([0], [1])
    r = random.Random(3)
    for c, first in ((1, 37), (0, 1), (1, 0)):
        now = pg.length(c)
        kept = sorted(r.sample(range(now - first), (now - first) * 2 // 3))
        before = [x.cpu() for x in pg.read([c], [0], [now])]
        pg.compact([c], [first], [kept])
        at = torch.tensor(list(range(first)) + [first + j for j in kept])
        for got, was in zip(pg.read([c], [0], [len(at)]), before):
            assert torch.equal(got.cpu(), was[:, at])
    # a tree's rows, of many clients at once
    pg.truncate([0, 1, 2], [0, 0, 0])


# ---- attention -----------------------------------------------------------------------------------


def attend_case(nq, nkv, dim, dtype, before, rows, trees=None, seed=0, scale=1.0, spoil=None):
    """Runs a pass of rows[i] rows behind before[i] tokens and compares it.  spoil(client, k, v): changes keys and values."""
    shape = shape_of(nq, nkv, dim, dtype, layers=2)
    n = len(before)
    pg = make_cache(shape, n, sum(-(-(b + r) // 16) for b, r in zip(before, rows)) + 3)
    ks, vs = ([random_rows(b + r, nkv, dim, dtype, seed + 10 * c + j) for c, (b, r) in enumerate(zip(before, rows))] for j in (1, 2))
    for c in range(n):
        if spoil:
            spoil(c, ks[c], vs[c])
    order = list(range(n))
    random.Random(seed).shuffle(order)
    for c in order:
        fill(pg, 1, c, ks[c], vs[c], before[c])
    flat = None if trees is None else [p for t in trees for p in t]
    pg.extend(list(range(n)), rows, flat)
    pg.append(1, torch.cat([k[b:] for k, b in zip(ks, before)]).cuda(), torch.cat([v[b:] for v, b in zip(vs, before)]).cuda())
    q = random_rows(sum(rows), nq, dim, dtype, seed + 7, scale)
    out = pg.attend(1, q.cuda())
    again = pg.attend(1, q.cuda())
    r = 0
    for c in range(n):
        parents = trees[c] if trees else list(range(-1, rows[c] - 1))
        want = reference(q[r:r + rows[c]], ks[c], vs[c], sees(before[c], parents))
        check_rows(out[r:r + rows[c]], *want, dtype)
        r += rows[c]
    assert torch.equal(out.nan_to_num(7), again.nan_to_num(7))
    return pg, q, out


HEADS = [(4, 4, 64), (8, 2, 128), (6, 2, 64), (8, 1, 128), (48, 3, 64)]


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("before", [0, 1, 15, 16, 33, 300])
def test_trees_behind_short_texts(heads, before, dtype):
    for rows in (1, 2, 5, 17):
        attend_case(*heads, dtype, [before], [rows], [random_tree(rows, rows, roots=before > 0)], seed=rows)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [(8, 2, 128), (6, 2, 64)])
def test_large_trees(heads, dtype):
    for before, rows in ((31, 256), (0, 255), (64, 33), (1000, 64), (127, 130)):
        attend_case(*heads, dtype, [before], [rows], [random_tree(rows, rows)], seed=before)
    attend_case(*heads, dtype, [77], [200], [[-1] * 200], seed=5)  # rows that see the text and themselves
    attend_case(*heads, dtype, [0], [40], [[-1] * 40], seed=6)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_chains(dim, dtype):
    for before, rows in ((0, 1), (0, 33), (100, 31), (511, 1), (3000, 9), (5, 400), (900, 600)):
        attend_case(8, 2, dim, dtype, [before], [rows], seed=before + rows)


@gpu
def test_a_chain_of_parents_is_a_chain():
    pg, q, out = attend_case(8, 2, 128, "bf16", [333, 20], [9, 4], [list(range(-1, 8)), list(range(-1, 3))])
    _, _, same = attend_case(8, 2, 128, "bf16", [333, 20], [9, 4])
    assert torch.equal(out, same)
    _, _, tree = attend_case(8, 2, 128, "bf16", [333, 20], [9, 4], [list(range(-1, 8)), [-1, 0, 1, 1]])
    assert torch.equal(out[:12], tree[:12])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [(8, 2, 128), (16, 16, 64), (24, 8, 128)])
def test_ragged_clients(heads, dtype):
    r = random.Random(1)
    before = [0, 1, 4000, 17, 800, 64, 2500, 333, 1200]
    rows = [3, 1, 17, 40, 2, 64, 9, 1, 33]
    attend_case(*heads, dtype, before, rows, [random_tree(n, n) for n in rows])
    before = [r.randint(0, 500) for _ in range(40)]
    rows = [r.randint(1, 20) for _ in range(40)]
    attend_case(*heads, dtype, before, rows, [random_tree(n, n, roots=True) for n in rows], seed=3)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_long_contexts(dim, dtype):
    attend_case(8, 2, dim, dtype, [40000], [5], [random_tree(5, 1)])
    attend_case(4, 1, dim, dtype, [70001, 12], [33, 3], [random_tree(33, 1), random_tree(3, 2)], seed=1, scale=2.0)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_does_not_reach_it(bad, dim, dtype):
    """Keys or values of drafts that are no numbers: rows of other branches are as if they were not there, rows that see them have what
    the definition gives."""
    before, rows = [50, 7], [40, 9]
    trees = [random_tree(n, 11 + n, roots=True) for n in rows]

    def spoil_values(c, k, v):
        for row in (3, 20) if c == 0 else (4,):
            v[before[c] + row, 1, 5 + row] = bad
            v[before[c] + row, 0, 40] = bad

    def spoil_keys(c, k, v):
        for row in (3, 20) if c == 0 else (4,):
            k[before[c] + row, 1, 5 + row] = bad

    for spoil in (spoil_values, spoil_keys):
        _, _, out = attend_case(8, 2, dim, dtype, before, rows, trees, spoil=spoil)
        assert not torch.isfinite(out).all() and torch.isfinite(out).any()
    attend_case(8, 2, dim, dtype, before, rows, spoil=spoil_values)  # chains
    # of the text, which all see
    attend_case(8, 2, dim, dtype, [50], [6], [[-1, 0, 0, 1, 1, 2]], spoil=lambda c, k, v: v[20, 1].fill_(bad))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_wider_matrices_and_results_in_place(dtype):
    nq, nkv, dim = 8, 2, 128
    pg, q, out = attend_case(nq, nkv, dim, dtype, [200, 1500], [9, 33], [random_tree(9, 1), random_tree(33, 2)])
    rows = q.shape[0]
    wide = torch.full((rows + 2, 2 * nq * dim + 64), 7.0, dtype=q.dtype, device="cuda")
    wide[:rows, :nq * dim] = q.flatten(1).cuda()
    pg.attend(1, wide[:rows, :nq * dim], out=wide[:rows, nq * dim + 64:])
    assert torch.equal(wide[:rows, nq * dim + 64:], out.flatten(1))
    assert bool((wide[rows:] == 7).all()) and bool((wide[:rows, nq * dim:nq * dim + 64] == 7).all())
    pg.attend(1, wide[:rows, :nq * dim], out=wide[:rows, :nq * dim])
    assert torch.equal(wide[:rows, :nq * dim], out.flatten(1))
    with pytest.raises(nav.PipesdError):
        pg.attend(1, wide[:rows, :nq * dim], out=wide[1:rows + 1, :nq * dim])
    with pytest.raises(TypeError):
        pg.attend(1, q)
    with pytest.raises(ValueError):
        pg.attend(1, q.cuda()[1:])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_forked_clients_attend_to_the_shared_text(dtype):
    nq, nkv, dim, n = 8, 2, 64, 141
    pg = make_cache(shape_of(nq, nkv, dim, dtype), 4, 40)
    k, v = (random_rows(n, nkv, dim, dtype, j) for j in (1, 2))
    fill(pg, 0, 0, k, v, n)
    pg.fork([0, 0, 0], [1, 2, 3], [n, n, 100])
    free = pg.free_blocks()
    rows = [5, 3, 7, 9]
    trees = [random_tree(m, m) for m in rows]
    pg.extend([2, 0, 3, 1], rows, [p for t in trees for p in t])
    # a last block of their own for 2, 0 and 3 (1 keeps the one that the others had, too), another for the 146 and 150 tokens of 2 and 1
    assert free - pg.free_blocks() == 5
    nk, nv, q = (random_rows(sum(rows), h, dim, dtype, j) for h, j in ((nkv, 3), (nkv, 4), (nq, 5)))
    pg.append(0, nk.cuda(), nv.cuda())
    out = pg.attend(0, q.cuda())
    r = 0
    for m, tree, had in zip(rows, trees, (n, n, 100, n)):
        want = reference(q[r:r + m], torch.cat([k[:had], nk[r:r + m]]), torch.cat([v[:had], nv[r:r + m]]), sees(had, tree))
        check_rows(out[r:r + m], *want, dtype)
        r += m


@gpu
def test_a_recorded_pass():
    """A layer's append and attend recorded with a tree, and replayed on other rows; eager passes between the replays."""
    nq, nkv, dim, before, rows = 8, 2, 128, 700, 21
    pg = make_cache(shape_of(nq, nkv, dim), 2, 120)
    k, v = (random_rows(before, nkv, dim, "bf16", j) for j in (1, 2))
    fill(pg, 0, 0, k, v, before)
    fill(pg, 0, 1, k, v, 33)
    tree = random_tree(rows, 4)
    nk, nv, q = (random_rows(rows, h, dim, "bf16", j).cuda() for h, j in ((nkv, 3), (nkv, 4), (nq, 5)))
    out = torch.empty_like(q)
    pg.extend([0], [rows], tree)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        pg.append(0, nk, nv)
        pg.attend(0, q, out=out)
        for call in (lambda: pg.extend([1], [3], [-1, 0, 0]), lambda: pg.fork([0], [1]), lambda: pg.copy([0], [1]),
                     lambda: pg.compact([1], [0], [[1, 2]])):
            with pytest.raises(nav.PipesdError) as e:
                call()
            assert e.value.status == nav.ESTATE
    assert pg.length(1) == 33
    for seed in range(10, 14):
        for x, h, j in ((nk, nkv, 3), (nv, nkv, 4), (q, nq, 5)):
            x.copy_(random_rows(rows, h, dim, "bf16", 10 * seed + j))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = reference(q.cpu(), torch.cat([k, nk.cpu()]), torch.cat([v, nv.cpu()]), sees(before, tree))
        check_rows(out, *want, "bf16")
        pg.extend([1], [4])  # (a chain: the tree's masks stay)
        x = random_rows(4, nkv, dim, "bf16", seed).cuda()
        pg.append(0, x, x)
        pg.attend(0, random_rows(4, nq, dim, "bf16", seed).cuda())


@gpu
def test_what_ends_a_pass():
    nq, nkv, dim = 4, 2, 64
    pg = make_cache(shape_of(nq, nkv, dim), 4, 40)
    k = random_rows(30, nkv, dim, "bf16", 1).cuda()
    q = random_rows(30, nq, dim, "bf16", 1).cuda()

    def begin():
        pg.truncate([0, 1, 2], [0, 0, 0])
        pg.extend([0, 1], [20, 10])
        pg.append(0, k, k)

    def closed():
        with pytest.raises(nav.PipesdError) as e:
            pg.attend(0, q)
        assert e.value.status == nav.ESTATE

    begin()
    pg.fork([0], [2])
    pg.compact([0], [10], [list(range(10))])
    pg.truncate([1], [10])
    pg.attend(0, q)
    for end in (lambda: pg.truncate([1], [9]), lambda: pg.compact([0], [10], [[1]]), lambda: pg.fork([0], [1]), lambda: pg.copy([1], [0])):
        begin()
        end()
        closed()
