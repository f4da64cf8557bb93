"""The cache held in 4 bits against its definition in 64 bits: what rows are stored as, attention over it (causal and limited
rows, ragged clients, both dtypes and head sizes, few and many rows, short and long contexts), the weights given to cached
tokens, cuts, and what is refused.  The pool starts as bytes of ones, so whatever is read beyond a client's tokens is not a
number.

Bounds, set before the first run.  A row o = sum p v, with S = sum p |v| and A = the largest sum |q k| / sqrt(d) of its row:
 * scores: 128 products in up to 5 pieces, summed in fp32 in some order: rounding errors of 2^-24 that add like a random
   walk over 640 sums are 2^-19 of sum |q k|, twice that allowed; an error of a score is the relative error of its weight: 2^-18 A;
 * bf16: results are rounded to 8 bits: 2^-8 |o| <= 2^-8 S (weights have 16 bits, well within it);
 * fp32: weights are cut to 16 bits or more: 2^-17 S, which also covers the fp32 sums over the tokens;
 * weights below the smallest normal fp32 number may be lost: their sum is below 2^-100;
 * the weight of a token: 2^-18 (1 + A) of it.
What is stored, kept and moved is compared exactly."""
import math

import pytest
import torch

from paper_2605_13319_amd import inputs as I
from paper_2605_13319_amd import nav

gpu = pytest.mark.gpu
GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def shape_of(nq, nkv, dim, dtype="bf16", layers=1):
    return I.ModelShape("kv4", layers, 512, nq, nkv, dim, 512, 512, dtype=I.DTYPE_F32 if dtype == "f32" else I.DTYPE_BF16)


def make_cache(shape, max_seqs, tokens):
    kv = nav.KV4Cache(shape, max_seqs, max_seqs * -(-tokens // 16))
    kv.pool.fill_(255)
    return kv


def held(x):
    """What the format holds for x [..][dim], by the definition, in 64 bits."""
    x = x.detach().cpu().double()
    x = torch.where(torch.isnan(x), 0.0, x).clamp(-3.4028234663852886e38, 3.4028234663852886e38).unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)  # top = m 2^e, m in [0.5, 1): <= 7 2^(e - 3) iff m <= 0.875
    e = torch.where(m <= 0.875, e - 3, e - 2)
    e = torch.where(top > 0, e, torch.full_like(e, -125)).clamp(-125, 125)
    power = torch.ldexp(torch.ones_like(top), e)
    a = (x.abs() / power).clamp(max=6)
    d = (a.unsqueeze(-1) - GRID).abs()
    low = d.argmin(-1)  # the lower of two equally near ones; of those the even one is meant
    tie = (low < 7) & (d.gather(-1, low.unsqueeze(-1)).squeeze(-1) == d.gather(-1, (low + 1).clamp(max=7).unsqueeze(-1)).squeeze(-1))
    code = torch.where(tie & (low % 2 == 1), low + 1, low)
    return (torch.sign(x) * GRID[code] * power).flatten(-2)


def reference(q, k, v, limits):
    """(o, S, A, weights) of one client: q [rows][nq][d]; k, v [tokens][nkv][d] as held, all 64 bits."""
    rows, nq, dim = q.shape
    tokens, nkv, _ = k.shape
    group = nq // nkv
    z = torch.einsum("rhgd,thd->hrgt", q.view(rows, nkv, group, dim), k) / math.sqrt(dim)
    sees = torch.arange(tokens)[None, :] < torch.as_tensor(limits)[:, None]
    big = torch.einsum("rhgd,thd->hrgt", q.view(rows, nkv, group, dim).abs(), k.abs()) / math.sqrt(dim)
    big = big.masked_fill(~sees[None, :, None], 0).amax(-1)
    p = torch.nan_to_num(torch.softmax(z.masked_fill(~sees[None, :, None], -torch.inf), -1))
    o = torch.einsum("hrgt,thd->rhgd", p, v).reshape(rows, nq, dim)
    s = torch.einsum("hrgt,thd->rhgd", p, v.abs()).reshape(rows, nq, dim)
    return o, s, big.permute(1, 0, 2).reshape(rows, nq, 1), p.sum((1, 2)), big.amax((1, 2))


def random_rows(rows, heads, dim, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, heads, dim, generator=g) * scale
    x = x * (1 + 3 * (torch.rand(heads, dim, generator=g) < 0.05))
    return x.to(torch.float32 if dtype == "f32" else torch.bfloat16)


def check_rows(got, want, s, a, dtype):
    err = (got.cpu().double() - want).abs()
    bound = ((2.0 ** -17 if dtype == "f32" else 2.0 ** -8) + 2.0 ** -18 * a) * s + 2.0 ** -100
    worst = float((err - bound).max())
    assert worst <= 0, (worst, float(err.max()))


# ---- store and read ------------------------------------------------------------------------------


def edge_rows(dim, dtype):
    """Rows with values on the borders of the rounding, blocks of zeros, the largest and smallest powers, NaN and infinities."""
    g = torch.Generator().manual_seed(5)
    rows = []
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 6.5, 7, 0.2501, 0.7499, 0, -0.25, -0.75, -7])
    for power in (0, 1, -1, 30, -30, 119, 120, -118, -119, -120, -123):
        x = torch.ldexp(ties.repeat(dim // 16), torch.tensor(power))
        rows += [x, torch.roll(x, 3) * 0.96875]
    for top in (6.98, 7.0, 7.03, 3.5, 3.53):
        x = torch.rand(dim, generator=g) * top
        x[::32] = top
        rows.append(x)
    x = torch.randn(dim, generator=g)
    x[5], x[40] = torch.nan, torch.inf
    rows += [torch.zeros(dim), x, -x, torch.full((dim,), torch.nan), torch.full((dim,), -torch.inf), torch.randn(dim, generator=g) * 1e-39,
             torch.randn(dim, generator=g) * 1e-37, torch.full((dim,), 3e38)]
    return torch.stack(rows).to(torch.float32 if dtype == "f32" else torch.bfloat16)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_rows_are_held_as_the_format_says(dim, dtype):
    heads = 3
    x = edge_rows(dim, dtype)
    k = torch.stack([x, x.flip(0), x.roll(5, 0)], 1).contiguous()
    v = torch.stack([x.roll(7, 0), x, x.flip(0)], 1).contiguous()
    kv = make_cache(shape_of(3, heads, dim, dtype, layers=2), 1, len(x))
    kv.extend([0], [len(x)])
    kv.append(1, k.cuda(), v.cuda())
    gk, gv = kv.read([0], [0], [len(x)], layer0=1)
    assert torch.equal(gk[0].cpu().double(), held(k))
    assert torch.equal(gv[0].cpu().double(), held(v))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nkv,dim", [(1, 128), (8, 64), (5, 128)])
def test_ragged_passes_keep_every_client_apart(nkv, dim, dtype):
    shape = shape_of(nkv * 2, nkv, dim, dtype, layers=3)
    kv = make_cache(shape, 5, 120)
    want = {c: [[], []] for c in range(5)}
    for step, (ids, ns) in enumerate([([0, 1, 2], [1, 17, 40]), ([4, 2], [3, 1]), ([1, 0, 3, 4], [16, 0, 15, 29]), ([2], [50])]):
        n = sum(ns)
        kv.extend(ids, ns)
        parts = []
        for layer in range(3):
            k, v = (random_rows(n, nkv, dim, dtype, 100 * step + 10 * layer + j) for j in (0, 1))
            wide = torch.empty(n, 2 * nkv * dim + 16, dtype=k.dtype, device="cuda")  # rows of a wider matrix, as fused projections leave them
            wide[:, :nkv * dim], wide[:, nkv * dim + 16:] = k.flatten(1).cuda(), v.flatten(1).cuda()
            kv.append(layer, wide[:, :nkv * dim], wide[:, nkv * dim + 16:])
            parts.append((held(k), held(v)))
        r = 0
        for c, m in zip(ids, ns):
            for j in (0, 1):
                want[c][j].append(torch.stack([p[j][r:r + m] for p in parts]))
            r += m
    ids = [3, 0, 2, 1, 4]
    lens = [kv.length(c) for c in ids]
    assert lens == [15, 1, 91, 33, 32]
    gk, gv = kv.read(ids, [0] * 5, lens)
    for j, got in enumerate((gk, gv)):
        assert torch.equal(got.cpu().double(), torch.cat([torch.cat(want[c][j], 1) for c in ids], 1))
    gk, _ = kv.read([2, 1], [13, 32], [30, 1], layer0=1, n_layers=1)
    assert torch.equal(gk.cpu().double(), torch.cat([torch.cat(want[2][0], 1)[1:2, 13:43], torch.cat(want[1][0], 1)[1:2, 32:33]], 1))
    assert kv.read([0], [1], [0])[0].shape == (3, 0, nkv, dim)


# ---- attention -----------------------------------------------------------------------------------


def attend_case(nq, nkv, dim, dtype, before, rows, limits=None, mass=None, seed=0, scale=1.0, chunk=700):
    """Runs a pass of rows[i] rows behind before[i] tokens and compares it; limits: a function (client, row, own) -> int."""
    shape = shape_of(nq, nkv, dim, dtype, layers=2)
    most = max(b + r for b, r in zip(before, rows))
    kv = make_cache(shape, len(before), most)
    ks, vs = ([random_rows(b + r, nkv, dim, dtype, seed + 10 * c + j) for c, (b, r) in enumerate(zip(before, rows))] for j in (1, 2))
    for c, b in enumerate(before):
        for f in range(0, b, chunk):
            n = min(chunk, b - f)
            kv.extend([c], [n])
            kv.append(1, ks[c][f:f + n].cuda(), vs[c][f:f + n].cuda())
    ids = list(range(len(before)))
    kv.extend(ids, rows)
    kv.append(1, torch.cat([k[b:] for k, b in zip(ks, before)]).cuda(), torch.cat([v[b:] for v, b in zip(vs, before)]).cuda())
    q = random_rows(sum(rows), nq, dim, dtype, seed + 7, scale)
    lim = [[b + i + 1 if limits is None else limits(c, i, b + i + 1) for i in range(r)] for c, (b, r) in enumerate(zip(before, rows))]
    flat = torch.tensor([x for c in lim for x in c], dtype=torch.int32).cuda() if limits else None
    weights = None if mass is None else torch.full((len(before), 2, nkv, most + 3), torch.nan, device="cuda")
    if mass:
        weights.fill_(2.0)
    out = kv.attend(1, q.cuda(), limits=flat, mass=weights, decay=mass or 0.0)
    again = kv.attend(1, q.cuda(), limits=flat)
    torch.cuda.synchronize()
    assert torch.equal(out, again) or torch.isnan(out).any()
    r = 0
    for c, (b, n) in enumerate(zip(before, rows)):
        if n == 0:
            continue
        seen = [min(max(x, 0), b + n) for x in lim[c]]
        o, s, a, w, big = reference(q[r:r + n].double(), held(ks[c]), held(vs[c]), seen)
        check_rows(out[r:r + n], o, s, a, dtype)
        if weights is not None:
            got = weights[c, 1].cpu().double()
            w = w + torch.where(torch.arange(b + n) < b, 2.0 * (mass or 0.0), 0.0)
            bound = 2.0 ** -18 * (1 + big[:, None]) * w + 1e-30
            assert bool(((got[:, :b + n] - w).abs() <= bound).all()), float(((got[:, :b + n] - w).abs() / w.clamp(min=1e-30)).max())
            left = got[:, b + n:]
            assert bool((left == 2.0).all() if mass else torch.isnan(left).all())
        r += n
    return kv


HEADS = [(4, 4, 64), (8, 2, 64), (6, 2, 128), (7, 1, 128), (16, 2, 64), (32, 8, 128)]


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("before,rows", [(0, 1), (0, 2), (14, 1), (15, 1), (15, 2), (16, 1), (30, 3), (31, 1), (0, 33), (100, 9), (127, 2),
                                         (500, 17), (1001, 5), (3000, 1)])
def test_one_client(heads, before, rows, dtype):
    print("case", heads, before, rows, dtype, flush=True)
    attend_case(*heads, dtype, [before], [rows], seed=before + rows, scale=1.5)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,before,rows", [((8, 2, 64), 77, 64), ((8, 2, 64), 0, 300), ((6, 2, 128), 500, 129), ((32, 8, 128), 40, 70),
                                               ((4, 4, 64), 1000, 257), ((7, 1, 128), 3, 333), ((8, 1, 128), 2500, 200)])
def test_many_rows(heads, before, rows, dtype):
    print("case", heads, before, rows, dtype, flush=True)
    attend_case(*heads, dtype, [before], [rows], seed=before + rows)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [(8, 2, 64), (6, 2, 128)], ids=str)
def test_ragged_clients(heads, dtype):
    attend_case(*heads, dtype, [0, 900, 33, 200, 15, 1], [1, 3, 17, 0, 5, 32])


@gpu
def test_few_and_many_rows_in_one_pass():
    attend_case(8, 2, 64, "bf16", [10, 700, 3], [1, 200, 9])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,before,rows", [((8, 2, 64), [600, 20], [9, 70]), ((6, 2, 128), [300, 0], [40, 3]), ((4, 4, 64), [60], [300])])
def test_rows_that_see_less_than_their_text_or_nothing(heads, before, rows, dtype):
    def limits(c, i, own):
        return [own, 0, own // 2, 1, -5, own + 1000, 16, 33][(i + c) % 8]
    attend_case(*heads, dtype, before, rows, limits=limits, mass=None, seed=3)
    attend_case(*heads, dtype, before, rows, limits=limits, mass=0.0, seed=4)
    attend_case(*heads, dtype, before, rows, limits=lambda c, i, own: 0, mass=0.5, seed=5)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,before,rows", [((8, 2, 64), [0], [1]), ((6, 2, 128), [500, 31, 0], [9, 1, 17]), ((16, 2, 64), [1200], [100]),
                                               ((4, 4, 64), [40], [333])])
@pytest.mark.parametrize("decay", [0.0, 0.75, 1.0])
def test_weights_given_to_cached_tokens(heads, before, rows, dtype, decay):
    attend_case(*heads, dtype, before, rows, mass=decay, seed=11)


@gpu
def test_a_context_of_more_than_32768_tokens():
    attend_case(4, 1, 64, "bf16", [40000], [2], mass=0.0, seed=21, chunk=20000)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_peaked_and_large_scores(dtype):
    """Scores of hundreds: one token takes nearly all weight, and the running maximum jumps."""
    attend_case(6, 2, 128, dtype, [700], [9], scale=40.0, seed=31)
    attend_case(8, 2, 64, dtype, [300], [100], scale=40.0, seed=32)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_and_nan_reach_only_the_rows_that_have_them(dtype):
    dim, nq, nkv = 128, 4, 2
    kv = make_cache(shape_of(nq, nkv, dim, dtype), 1, 64)
    k, v, q = (random_rows(50, h, dim, dtype, s) for h, s in ((nkv, 1), (nkv, 2), (nq, 3)))
    k[30, 0, 7], v[31, 1, 9], v[32, 0, 0] = torch.nan, torch.inf, -torch.inf
    q[10, 1, 3], q[20, 2, 5] = torch.nan, -torch.inf
    kv.extend([0], [50])
    kv.append(0, k.cuda(), v.cuda())
    lim = [1 + i % 30 for i in range(50)]
    out = kv.attend(0, q.cuda(), limits=torch.tensor(lim, dtype=torch.int32).cuda()).cpu()
    bad = torch.isnan(out).all(-1)
    assert torch.equal(bad, torch.isnan(out).any(-1))
    want = torch.zeros(50, nq, dtype=torch.bool)
    want[10, 1] = want[20, 2] = True
    assert torch.equal(bad, want)
    q[10, 1, 3] = q[20, 2, 5] = 0
    o, s, a, _, _ = reference(q.double(), held(k), held(v), lim)
    good = ~want
    check_rows(out[good], o[good], s[good], a[good], dtype)


@gpu
def test_rows_of_wider_matrices_and_another_stream():
    nq, nkv, dim, n = 8, 2, 128, 19
    kv = make_cache(shape_of(nq, nkv, dim), 1, 64)
    k, v, q = (random_rows(n, h, dim, "bf16", s) for h, s in ((nkv, 1), (nkv, 2), (nq, 3)))
    wide = torch.randn(n, (nq + 2 * nkv) * dim).bfloat16().cuda()
    wide[:, :nq * dim], wide[:, nq * dim:(nq + nkv) * dim], wide[:, (nq + nkv) * dim:] = q.flatten(1).cuda(), k.flatten(1).cuda(), v.flatten(1).cuda()
    out = torch.full((n, 2 * nq * dim), 7.0, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        kv.extend([0], [n])
        kv.append(0, wide[:, nq * dim:(nq + nkv) * dim], wide[:, (nq + nkv) * dim:])
        kv.attend(0, wide[:, :nq * dim], out=out[:, nq * dim:])
    torch.cuda.current_stream().wait_stream(side)
    assert bool((out[:, :nq * dim] == 7.0).all())
    o, s, a, _, _ = reference(q.double(), held(k), held(v), list(range(1, n + 1)))
    check_rows(out[:, nq * dim:].view(n, nq, dim), o, s, a, "bf16")


@gpu
def test_a_clients_rows_do_not_depend_on_who_shares_the_pass():
    """(of passes with the same most rows)"""
    nq, nkv, dim = 8, 2, 64
    kv = make_cache(shape_of(nq, nkv, dim), 4, 600)
    ks = [random_rows(500, nkv, dim, "bf16", 40 + c) for c in range(4)]
    kv.extend([0, 1, 2, 3], [490] * 4)
    kv.append(0, torch.cat([k[:490] for k in ks]).cuda(), torch.cat([k[:490] for k in ks]).cuda())
    q = random_rows(40, nq, dim, "bf16", 9).cuda()
    new = torch.cat([k[490:] for k in ks]).cuda()
    kv.extend([0, 1, 2, 3], [10] * 4)
    kv.append(0, new, new)
    all_four = kv.attend(0, q)
    for c in range(4):
        kv.truncate([c], [490])
        kv.extend([c], [10])
        kv.append(0, new[10 * c:10 * c + 10], new[10 * c:10 * c + 10])
        assert torch.equal(kv.attend(0, q[10 * c:10 * c + 10]), all_four[10 * c:10 * c + 10])


@gpu
def test_recorded_in_a_graph():
    """One decoding step's launches, replayed on new queries, keys and values."""
    nq, nkv, dim = 8, 2, 128
    kv = make_cache(shape_of(nq, nkv, dim), 1, 800)
    ks, vs = random_rows(700, nkv, dim, "bf16", 1), random_rows(700, nkv, dim, "bf16", 2)
    kv.extend([0], [699])
    kv.append(0, ks[:699].cuda(), vs[:699].cuda())
    k, v = torch.zeros(1, nkv, dim, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, nkv, dim, dtype=torch.bfloat16, device="cuda")
    q, out = torch.zeros(1, nq, dim, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, nq, dim, dtype=torch.bfloat16, device="cuda")
    weights = torch.zeros(1, 1, nkv, 800, device="cuda")
    kv.extend([0], [1])
    kv.append(0, k, v)
    kv.attend(0, q, out=out, mass=weights, decay=0.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv.append(0, k, v)
        kv.attend(0, q, out=out, mass=weights, decay=0.0)
    for i in range(4):
        nk, nv, nq_ = (random_rows(1, h, dim, "bf16", 50 + 3 * i + j) for j, h in enumerate((nkv, nkv, nq)))
        k.copy_(nk), v.copy_(nv), q.copy_(nq_)
        graph.replay()
        torch.cuda.synchronize()
        o, s, a, w, big = reference(nq_.double(), torch.cat([held(ks[:699]), held(nk)]), torch.cat([held(vs[:699]), held(nv)]), [700])
        check_rows(out, o, s, a, "bf16")
        assert bool(((weights[0, 0, :, :700].cpu().double() - w).abs() <= 2.0 ** -18 * (1 + big[:, None]) * w).all())
        torch.zeros(1 << 20, device="cuda").add_(1).sum().item()  # other work between the replays


# ---- cuts ----------------------------------------------------------------------------------------


def chosen(w, keep, recent):
    """Indices that stay, of one layer and head: a list sorted in plain Python."""
    n = len(w)
    w = [0.0 if x != x else x for x in w]
    order = sorted(range(n - recent), key=lambda t: (-w[t], t))[:keep - recent]
    return sorted(order) + list(range(n - recent, n))


@gpu
@pytest.mark.parametrize("dtype,nkv,dim", [("bf16", 2, 64), ("f32", 3, 128)])
@pytest.mark.parametrize("length,keep,recent", [(1, 1, 0), (1, 1, 1), (17, 16, 3), (40, 40, 7), (40, 1, 1), (40, 1, 0), (300, 33, 33), (300, 299, 0),
                                                (4500, 1000, 64), (9000, 4097, 1)])
@pytest.mark.parametrize("in_place", [False, True])
def test_cuts(dtype, nkv, dim, length, keep, recent, in_place):
    layers = 2
    shape = shape_of(nkv, nkv, dim, dtype, layers)
    kv = nav.KV4Cache(shape, 3, 3 * -(-length // 16) + -(-keep // 16))
    kv.pool.fill_(255)
    k, v = ([random_rows(length, nkv, dim, dtype, 60 + 2 * layer + j) for layer in range(layers)] for j in (0, 1))
    g = torch.Generator().manual_seed(length + keep)
    w = torch.rand(3, layers, nkv, length + 5, generator=g).pow(6)
    w[torch.rand(w.shape, generator=g) < 0.3] = 0.0            # many equal ones
    w = torch.where(torch.rand(w.shape, generator=g) < 0.2, (w * 16).round() / 16, w)
    w[1, 0, 0, ::7] = torch.nan
    w[1, 1, 0, 1::5] = -0.0
    kv.extend([0, 1, 2], [3, length, 2])
    for layer in range(layers):
        kv.append(layer, torch.cat([k[layer][:1].expand(3, -1, -1), k[layer], k[layer][:1].expand(2, -1, -1)]).cuda(),
                  torch.cat([v[layer][:1].expand(3, -1, -1), v[layer], v[layer][:1].expand(2, -1, -1)]).cuda())
    mass = w.cuda()
    into = 1 if in_place else 2
    free = kv.free_blocks()
    kept = kv.evict([1], [into], keep, recent, mass)
    assert kv.length(into) == keep and kv.seq_blocks(into) == -(-keep // 16)
    assert kv.length(1) == (keep if in_place else length) and kv.length(0) == 3
    assert kv.free_blocks() == free + (kv.seq_blocks(1) * 0 + -(-length // 16) if in_place else 1) - -(-keep // 16)
    gk, gv = kv.read([into], [0], [keep])
    for layer in range(layers):
        hk, hv = held(k[layer]), held(v[layer])
        for h in range(nkv):
            idx = chosen(w[1, layer, h, :length].tolist(), keep, recent)
            assert kept[0, layer, h].tolist() == idx, (layer, h)
            assert torch.equal(gk[layer, :, h].cpu().double(), hk[idx, h]) and torch.equal(gv[layer, :, h].cpu().double(), hv[idx, h])
            assert torch.equal(mass[into, layer, h, :keep].cpu().view(torch.int32), w[1, layer, h][idx].view(torch.int32))
    gk, _ = kv.read([0], [0], [3])
    assert torch.equal(gk[1].cpu().double(), held(k[1][:1].expand(3, -1, -1)))


@gpu
def test_a_cut_client_goes_on():
    """Rows appended behind a cut, attention over what is left, the weights of both; two clients cut at once."""
    nq, nkv, dim, layers = 6, 2, 64, 2
    kv = make_cache(shape_of(nq, nkv, dim, "bf16", layers), 2, 400)
    lens = [130, 200]
    ks, vs = ([random_rows(n + 5, nkv, dim, "bf16", 80 + 2 * c + j) for c, n in enumerate(lens)] for j in (0, 1))
    kv.extend([0, 1], lens)
    for layer in range(layers):
        kv.append(layer, torch.cat([k[:-5] for k in ks]).cuda(), torch.cat([v[:-5] for v in vs]).cuda())
    mass = torch.rand(2, layers, nkv, 400, generator=torch.Generator().manual_seed(1)).cuda()
    before = mass.cpu()
    kept = kv.evict([1, 0], [1, 0], 100, 10, mass).cpu()
    with pytest.raises(nav.PipesdError) as e:  # the pass is over
        kv.attend(0, torch.zeros(330, nq, dim, dtype=torch.bfloat16, device="cuda"))
    assert e.value.status == nav.ESTATE
    kv.extend([0, 1], [5, 5])
    q = random_rows(10, nq, dim, "bf16", 99)
    for layer in range(layers):
        kv.append(layer, torch.cat([k[-5:] for k in ks]).cuda(), torch.cat([v[-5:] for v in vs]).cuda())
        out = kv.attend(layer, q.cuda(), mass=mass, decay=1.0)
        for c in (0, 1):
            idx = kept[1 - c, layer].long()
            pick = lambda x: torch.cat([torch.gather(held(x[:-5]), 0, idx.T[..., None].expand(-1, -1, dim)), held(x[-5:])])  # noqa: E731
            o, s, a, w, big = reference(q[5 * c:5 * c + 5].double(), pick(ks[c]), pick(vs[c]), list(range(101, 106)))
            check_rows(out[5 * c:5 * c + 5], o, s, a, "bf16")
            old = torch.gather(before[c, layer], 1, idx).double()
            want = w + torch.cat([old, torch.zeros(nkv, 5, dtype=torch.float64)], 1)
            assert bool(((mass[c, layer, :, :105].cpu().double() - want).abs() <= 2.0 ** -18 * (1 + big[:, None]) * want + 2.0 ** -23).all())


@gpu
def test_a_full_pool_takes_a_cut_back_to_where_it_was():
    nkv, dim = 2, 64
    kv = nav.KV4Cache(shape_of(2, nkv, dim), 2, 6)
    k = random_rows(96, nkv, dim, "bf16", 1).cuda()
    kv.extend([0], [96])
    kv.append(0, k, k)
    mass = torch.rand(2, 1, nkv, 96, device="cuda")
    for into in (0, 1):
        with pytest.raises(nav.PipesdError) as e:
            kv.evict([0], [into], 17, 0, mass)
        assert e.value.status == nav.ENOMEM
    assert (kv.length(0), kv.length(1), kv.free_blocks()) == (96, 0, 0)
    assert torch.equal(kv.read([0], [0], [96])[0][0].cpu().double(), held(k))


# ---- refusals and bookkeeping (no device) --------------------------------------------------------


def host_cache(max_seqs=4, n_blocks=8, **kw):
    return nav.KV4Cache(shape_of(4, 2, 64, **kw), max_seqs, n_blocks, on_device=False)


def refused(status, f, *a):
    with pytest.raises(nav.PipesdError) as e:
        f(*a)
    assert e.value.status == status


def test_shapes_that_are_refused():
    import ctypes as C
    import dataclasses
    good = shape_of(4, 2, 64)
    for bad in (dict(head_dim=96), dict(head_dim=32), dict(n_q_heads=5), dict(n_kv_heads=0), dict(n_layers=0), dict(dtype=2)):
        cfg = nav.config_of(dataclasses.replace(good, **bad))
        assert nav._lib.pipesd_kv4_block_bytes(C.byref(cfg), 16) == 0
        h = C.c_void_p()
        assert nav._lib.pipesd_kv4_create(C.byref(cfg), 1, 16, None, 1 << 20, C.byref(h)) == nav.EINVAL
    cfg = nav.config_of(good)
    h = C.c_void_p()
    lib = nav._lib
    assert lib.pipesd_kv4_block_bytes(C.byref(cfg), 16) == 2 * 1088 and lib.pipesd_kv4_block_bytes(C.byref(cfg), 32) == 0
    assert lib.pipesd_kv4_create(C.byref(cfg), 0, 16, None, 1 << 20, C.byref(h)) == nav.EINVAL
    assert lib.pipesd_kv4_create(C.byref(cfg), 1, 16, None, 2175, C.byref(h)) == nav.EINVAL
    assert lib.pipesd_kv4_create(C.byref(cfg), 1, 8, None, 1 << 20, C.byref(h)) == nav.EINVAL
    assert lib.pipesd_kv4_create(C.byref(cfg), 1, 16, None, 2176 << 27, C.byref(h)) == nav.EINVAL   # 2^31 tokens
    assert lib.pipesd_kv4_create(C.byref(cfg), 1 << 20, 16, None, 2176 << 10, C.byref(h)) == nav.EINVAL  # 2^31 table entries
    assert lib.pipesd_kv4_create(C.byref(cfg), 1, 16, C.c_void_p(4096 + 16), 1 << 20, C.byref(h)) == nav.EINVAL
    assert lib.pipesd_kv4_create(None, 1, 16, None, 1 << 20, C.byref(h)) == nav.EINVAL
    assert lib.pipesd_kv4_create(C.byref(cfg), 1, 16, None, 1 << 20, None) == nav.EINVAL
    assert lib.pipesd_kv4_destroy(None) == nav.EINVAL


def test_bookkeeping_of_blocks():
    kv = host_cache()
    kv.extend([0, 2], [16, 17])
    assert (kv.seq_blocks(0), kv.seq_blocks(2), kv.free_blocks()) == (1, 2, 5)
    refused(nav.ENOMEM, kv.extend, [1, 0], [64, 32])
    assert (kv.length(0), kv.length(1), kv.free_blocks()) == (16, 0, 5)
    kv.extend([1, 0], [63, 16])
    assert kv.free_blocks() == 0
    kv.extend([1, 3], [1, 0])
    refused(nav.ENOMEM, kv.extend, [3], [1])
    kv.truncate([2, 1], [16, 0])
    assert (kv.length(2), kv.seq_blocks(2), kv.length(1), kv.free_blocks()) == (16, 1, 0, 5)
    kv.truncate([2], [0])
    kv.extend([3], [96])
    assert kv.free_blocks() == 0 and kv.length(3) == 96


def test_passes_that_are_refused():
    kv = host_cache()
    for ids, ns in (([0, 0], [1, 1]), ([4], [1]), ([-1], [1]), ([0], [-1]), ([0], [0]), ([0, 1], [0, 0]), ([0], [2 ** 31 - 1])):
        refused(nav.EINVAL, kv.extend, ids, ns)
    with pytest.raises(ValueError):
        kv.extend([0, 1], [1])
    assert nav._lib.pipesd_kv4_extend(None, 1, None, None, None) == nav.EINVAL
    assert nav._lib.pipesd_kv4_extend(kv.handle, 1, None, None, None) == nav.EINVAL
    refused(nav.ESTATE, kv.truncate, [0], [1])
    refused(nav.ESTATE, kv.truncate, [0], [-1])
    refused(nav.EINVAL, kv.truncate, [0, 0], [0, 0])
    refused(nav.EINVAL, kv.length, 4)
    refused(nav.EINVAL, kv.seq_blocks, -1)


def test_pointers_strides_and_states_that_are_refused():
    import ctypes as C
    lib = nav._lib
    kv = host_cache(layers=2)
    kv.extend([0], [20])
    p, odd = 1 << 20, (1 << 20) + 8
    row = 2 * 64
    ap = lambda *a: lib.pipesd_kv4_append(kv.handle, *a, None)  # noqa: E731
    assert ap(2, p, row, p, row) == ap(-1, p, row, p, row) == ap(0, None, row, p, row) == ap(0, p, row, None, row) == nav.EINVAL
    assert ap(0, odd, row, p, row) == ap(0, p, row - 8, p, row) == ap(0, p, row, p, row + 4) == nav.EINVAL
    assert ap(0, p, row, p, row) == nav.ESTATE  # (no pool)
    at = lambda layer=0, q=p, qs=256, lim=None, o=p, os_=256, m=None, ms=0, decay=1.0: lib.pipesd_kv4_attend(  # noqa: E731
        kv.handle, layer, q, qs, lim, o, os_, m, ms, decay, None)
    assert at(layer=2) == at(q=None) == at(o=None) == at(qs=255) == at(os_=128) == at(q=odd) == at(lim=p + 2) == at(m=p + 1) == nav.EINVAL
    assert at() == nav.ESTATE
    i32 = lambda *a: (C.c_int32 * len(a))(*a)  # noqa: E731
    rd = lambda ids, f, c, l0=0, nl=2, k=p, v=p: lib.pipesd_kv4_read(kv.handle, len(ids), i32(*ids), i32(*f), i32(*c), l0, nl, k, v, None)  # noqa: E731
    assert rd([4], [0], [1]) == rd([0], [-1], [1]) == rd([0], [0], [-1]) == rd([0], [0], [1], 1, 2) == rd([0], [0], [1], 0, 0) == nav.EINVAL
    assert rd([0], [0], [1], k=None) == rd([0], [0], [1], v=odd) == nav.EINVAL
    assert rd([0], [15], [6]) == rd([1], [0], [1]) == rd([0], [0], [20]) == nav.ESTATE
    ev = lambda ids, to, keep, recent, m=p, ms=64, kept=p: lib.pipesd_kv4_evict(kv.handle, len(ids), i32(*ids), i32(*to), keep, recent, m, ms, kept, None)  # noqa: E731
    kv.extend([1], [20])
    assert ev([0], [0], 0, 0) == ev([0], [0], 5, 6) == ev([0], [0], 5, -1) == ev([0], [4], 5, 1) == ev([0, 0], [0, 1], 5, 1) == nav.EINVAL
    assert ev([0, 1], [1, 0], 5, 1) == ev([0, 1], [2, 2], 5, 1) == ev([0], [0], 5, 1, m=None) == ev([0], [0], 5, 1, kept=None) == nav.EINVAL
    assert ev([0], [0], 5, 1, ms=19) == nav.EINVAL
    assert ev([0], [0], 21, 1) == ev([0], [0], 5, 1) == nav.ESTATE
    assert (kv.length(0), kv.length(1), kv.free_blocks()) == (20, 20, 4)


@gpu
def test_tensors_that_are_refused():
    kv = make_cache(shape_of(4, 2, 64, "bf16"), 2, 64)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    kv.extend([0], [3])
    kv.append(0, x, x)
    for bad in (x.float(), x.cpu()):
        with pytest.raises(TypeError):
            kv.append(0, bad, x)
    for bad in (x[:2], x.transpose(0, 1), x[:, :1], torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda")[:, :, :64], q):
        with pytest.raises(ValueError):
            kv.append(0, x, bad)
    refused(nav.EINVAL, kv.append, 0, torch.zeros(3, 132, dtype=torch.bfloat16, device="cuda")[:, :128], x)  # rows 264 bytes apart
    mass = torch.zeros(2, 1, 2, 64, device="cuda")
    for bad in (dict(limits=torch.zeros(3, device="cuda")), dict(limits=torch.zeros(2, dtype=torch.int32, device="cuda")), dict(mass=mass[:1]),
                dict(mass=mass.double()), dict(mass=mass[..., :50]), dict(out=torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(ValueError):
            kv.attend(0, q, **bad)
    refused(nav.EINVAL, lambda: kv.attend(0, q, mass=mass, decay=1.5))
    refused(nav.EINVAL, lambda: kv.attend(0, q, mass=mass, decay=float("nan")))
    refused(nav.EINVAL, lambda: kv.attend(0, q, mass=torch.zeros(2, 1, 2, 2, device="cuda")))
    kv.truncate([0], [2])
    refused(nav.ESTATE, lambda: kv.attend(0, q))
    kv.truncate([0], [0])
    big = nav.KV4Cache(shape_of(4, 2, 64), 1, 200)
    big.extend([0], [2049])
    rows = torch.zeros(2049, 256, dtype=torch.bfloat16, device="cuda")
    big.append(0, rows[:, :128], rows[:, 128:])
    refused(nav.ESTATE, lambda: big.attend(0, rows))
