"""Passes over the 4-bit cache that are large enough for the kernel of many tiles, against their definition in 64 bits: both
dtypes and head sizes, groups of heads that fill tiles unevenly, clients of few rows beside them, contexts in one piece and in
many, rows that see less than their text or nothing, weights given to cached tokens, and a recorded pass.  (Which kernel a pass
takes is the plan's: tests/test_kv4_plan.py checks these cases.)  The bounds are those of tests/test_gpu_kv4.py, and what is held
is what the cache reads back as, which is checked there."""
import math

import pytest
import torch

from paper_2605_13319_amd import nav
from tests.test_gpu_kv4 import check_rows, make_cache, shape_of

gpu = pytest.mark.gpu

# heads (query, cache, size), dtype, tokens before and rows of each client
CASES = {
    "128": ((64, 8, 128), "bf16", [7936], [256]),
    "64": ((32, 8, 64), "bf16", [3100], [1024]),
    "64_f32": ((32, 32, 64), "f32", [15000], [512]),
    "128_f32": ((32, 4, 128), "f32", [9000], [1024]),
    "group_of_7": ((7, 1, 128), "bf16", [7003], [2045]),
    "long": ((32, 8, 128), "bf16", [118001], [32]),
    "beside_few": ((32, 8, 64), "bf16", [5000, 3971, 100], [1, 1536, 3]),
    "two": ((32, 8, 64), "f32", [2999, 4200], [700, 601]),
    "prompt": ((24, 3, 64), "bf16", [0, 4080], [2048, 2048]),
}


def rows_of(n, heads, dim, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, heads, dim, generator=g, device="cuda")
    x = x * (1 + 3 * (torch.rand(heads, dim, generator=g, device="cuda") < 0.05))
    return x.to(torch.float32 if dtype == "f32" else torch.bfloat16)


def filled(name, seed):
    (nq, nkv, dim), dtype, before, rows = CASES[name]
    kv = make_cache(shape_of(nq, nkv, dim, dtype), len(before), max(b + r for b, r in zip(before, rows)))
    for c, b in enumerate(before):
        for f in range(0, b, 20000):
            n = min(20000, b - f)
            kv.extend([c], [n])
            kv.append(0, rows_of(n, nkv, dim, dtype, seed + 10 * c + f), rows_of(n, nkv, dim, dtype, seed + 10 * c + f + 1))
    kv.extend(list(range(len(before))), rows)
    n = sum(rows)
    kv.append(0, rows_of(n, nkv, dim, dtype, seed + 3), rows_of(n, nkv, dim, dtype, seed + 4))
    return kv, rows_of(n, nq, dim, dtype, seed + 5)


def definition(q, k, v, limits):
    """(o, S, A, weights, the largest A of a head) in 64 bits, a head of the cache at a time."""
    rows, nq, dim = q.shape
    tokens, nkv, _ = k.shape
    group = nq // nkv
    blind = torch.arange(tokens, device="cuda")[None] >= limits.repeat_interleave(group)[:, None]
    o, s = torch.empty(2, rows, nq, dim, dtype=torch.float64, device="cuda")
    a = torch.empty(rows, nq, 1, dtype=torch.float64, device="cuda")
    w = torch.empty(nkv, tokens, dtype=torch.float64, device="cuda")
    for h in range(nkv):
        qh = q[:, h * group:(h + 1) * group].double().reshape(-1, dim)
        kh, vh = k[:, h].double(), v[:, h].double()
        own = slice(h * group, (h + 1) * group)
        a[:, own] = (qh.abs() @ kh.abs().T.contiguous()).masked_fill_(blind, 0).amax(-1).view(rows, group, 1) / math.sqrt(dim)
        p = (qh @ kh.T.contiguous() / math.sqrt(dim)).masked_fill_(blind, -torch.inf).softmax(-1).nan_to_num_(0)
        o[:, own], s[:, own] = (p @ vh).view(rows, group, dim), (p @ vh.abs()).view(rows, group, dim)
        w[h] = p.sum(0)
    return o, s, a, w, a.view(rows, nkv, group).amax((0, 2))


def compare(name, kv, q, out, limits=None, mass=None):
    _, dtype, before, rows = CASES[name]
    r = 0
    for c, (b, n) in enumerate(zip(before, rows)):
        k, v = kv.read([c], [0], [b + n])
        own = torch.arange(b + 1, b + n + 1, device="cuda")
        o, s, a, w, big = definition(q[r:r + n], k[0], v[0], own if limits is None else limits[r:r + n].clamp(0, b + n))
        check_rows(out[r:r + n], o.cpu(), s.cpu(), a.cpu(), dtype)
        if mass is not None:
            bound = 2.0 ** -18 * (1 + big[:, None]) * w + 1e-30
            assert bool(((mass[c, 0, :, :b + n].double() - w).abs() <= bound).all())
            assert bool(torch.isnan(mass[c, 0, :, b + n:]).all())
        r += n


@gpu
@pytest.mark.parametrize("name", CASES)
def test_against_the_definition(name):
    print("case", name, flush=True)
    kv, q = filled(name, 100)
    out = kv.attend(0, q)
    assert torch.equal(kv.attend(0, q), out)
    compare(name, kv, q, out)


@gpu
@pytest.mark.parametrize("name", ["64", "64_f32", "128_f32", "long", "beside_few"])
def test_rows_that_see_less_or_nothing_and_the_weights_given(name):
    print("case", name, flush=True)
    kv, q = filled(name, 200)
    before, rows = CASES[name][2:]
    own = torch.cat([torch.arange(b + 1, b + n + 1) for b, n in zip(before, rows)])
    i = torch.arange(len(own))
    limits = torch.where(i % 9 == 0, 0, torch.where(i % 9 == 1, -3, torch.where(i % 9 == 2, own // 3, torch.where(i % 9 == 3, 1 + i % 70, own + i % 3))))
    limits[32:64] = 0  # a wave's rows all blind
    limits = limits.to(torch.int32).cuda()
    mass = torch.full((len(before), 1, kv.shape.n_kv_heads, max(b + n for b, n in zip(before, rows)) + 5), torch.nan, device="cuda")
    out = kv.attend(0, q, limits=limits, mass=mass, decay=0.0)
    compare(name, kv, q, out, limits, mass)


@gpu
@pytest.mark.parametrize("name", ["64", "128_f32"])
def test_peaked_scores_and_rows_of_infinities(name):
    """Scores of hundreds, larger the later the token: the running maximum moves again and again."""
    kv, q = filled(name, 300)
    before, rows = CASES[name][2:]
    q = q * 20
    bad = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    q[5, 1, 3], q[70, 2, 9], q[200, 0, 0] = torch.nan, torch.inf, -torch.inf
    bad[5, 1] = bad[70, 2] = bad[200, 0] = True
    out = kv.attend(0, q)
    assert torch.equal(torch.isnan(out).any(-1), bad) and torch.equal(torch.isnan(out).all(-1), bad)
    compare(name, kv, torch.where(bad[..., None], 0, q), torch.where(bad[..., None], kv.attend(0, torch.where(bad[..., None], 0, q)), out))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,rows", [(8, 9), (2, 1)])
def test_few_rows_of_nan_over_a_context_in_pieces(nq, rows, dtype):
    kv = make_cache(shape_of(nq, 2, 128, dtype), 1, 6000)
    kv.extend([0], [5000])
    kv.append(0, rows_of(5000, 2, 128, dtype, 1), rows_of(5000, 2, 128, dtype, 2))
    kv.extend([0], [rows])
    kv.append(0, rows_of(rows, 2, 128, dtype, 3), rows_of(rows, 2, 128, dtype, 4))
    q = rows_of(rows, nq, 128, dtype, 5)
    q[rows - 1, 1, 3] = torch.nan
    out = torch.isnan(kv.attend(0, q))
    assert bool(out[rows - 1, 1].all()) and int(out.sum()) == 128


@gpu
@pytest.mark.parametrize("name", ["128", "beside_few"])
def test_a_recorded_pass(name):
    kv, q = filled(name, 400)
    out = torch.empty_like(q)
    mass = torch.zeros(len(CASES[name][2]), 1, kv.shape.n_kv_heads, 9000, device="cuda")
    kv.attend(0, q, out=out, mass=mass, decay=0.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv.attend(0, q, out=out, mass=mass, decay=0.0)
    for seed in range(3):
        q.copy_(rows_of(*q.shape, "bf16", 500 + seed))
        other = torch.zeros_like(mass)
        want = kv.attend(0, q, mass=other, decay=0.0).clone()
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(mass, other)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_clients_than_a_launch_takes(dtype):
    """40 clients: rows kept, attention and weights of each, 35 of them cut at once."""
    n, nq, nkv, dim = 40, 8, 2, 64
    before, rows = [(37 * c) % 211 for c in range(n)], [(c * 5) % 9 for c in range(n)]
    kv = make_cache(shape_of(nq, nkv, dim, dtype), n, 240)
    held = [b > 0 for b in before]
    ids = [c for c in range(n) if held[c]]
    kv.extend(ids, [before[c] for c in ids])
    kv.append(0, rows_of(sum(before), nkv, dim, dtype, 1), rows_of(sum(before), nkv, dim, dtype, 2))
    kv.extend(list(range(n)), rows)
    total = sum(rows)
    kv.append(0, rows_of(total, nkv, dim, dtype, 3), rows_of(total, nkv, dim, dtype, 4))
    q = rows_of(total, nq, dim, dtype, 5)
    mass = torch.full((n, 1, nkv, 240), torch.nan, device="cuda")
    out = kv.attend(0, q, mass=mass, decay=0.0)
    r = 0
    for c, (b, m) in enumerate(zip(before, rows)):
        if m:
            k, v = kv.read([c], [0], [b + m])
            o, s, a, w, big = definition(q[r:r + m], k[0], v[0], torch.arange(b + 1, b + m + 1, device="cuda"))
            check_rows(out[r:r + m], o.cpu(), s.cpu(), a.cpu(), dtype)
            assert bool(((mass[c, 0, :, :b + m].double() - w).abs() <= 2.0 ** -18 * (1 + big[:, None]) * w + 1e-30).all())
        r += m
    cut = [c for c in range(n) if before[c] + rows[c] >= 20][:35]
    mass.nan_to_num_(0.0)
    old = [kv.read([c], [0], [before[c] + rows[c]]) for c in cut]
    weights = mass[cut, 0].cpu()
    kept = kv.evict(cut, cut, 20, 5, mass).cpu().long()
    k, v = kv.read(cut, [0] * len(cut), [20] * len(cut))
    assert len(cut) > 32
    for i, c in enumerate(cut):
        length = before[c] + rows[c]
        heavy = torch.argsort(-weights[i, :, :length - 5], dim=-1, stable=True)[:, :15].sort(-1).values
        want = torch.cat([heavy, torch.arange(length - 5, length).expand(nkv, 5)], -1)
        assert torch.equal(kept[i, 0], want)
        at = want.T[..., None].expand(-1, -1, dim).cuda()
        for new, was in ((k, old[i][0]), (v, old[i][1])):
            assert torch.equal(new[0, 20 * i:20 * i + 20], was[0].gather(0, at))


@gpu
def test_a_context_beyond_the_workgroups_of_a_grid():
    """8.5 million tokens whose keys are 0: the weights are all alike, and a cut keeps the first and the newest."""
    length, keep, recent = 8500000, 4300000, 100
    kv = nav.KV4Cache(shape_of(2, 1, 64), 1, -(-(length + 2) // 16) + -(-keep // 16))
    kv.pool.zero_()
    kv.extend([0], [length])
    kv.extend([0], [2])
    zero = torch.zeros(2, 1, 64, dtype=torch.bfloat16, device="cuda")
    kv.append(0, zero, rows_of(2, 1, 64, "bf16", 1))
    mass = torch.full((1, 1, 1, length + 2), torch.nan, device="cuda")
    out = kv.attend(0, rows_of(2, 2, 64, "bf16", 2), mass=mass, decay=0.0)
    assert float(out.abs().max()) < 1e-5
    want = torch.full((length + 2,), 2 / (length + 1) + 2 / (length + 2), dtype=torch.float64, device="cuda")
    want[-1] = 2 / (length + 2)
    assert bool(((mass[0, 0, 0].double() - want).abs() <= 2.0 ** -18 * want).all())
    mass.fill_(1.0)
    kept = kv.evict([0], [0], keep, recent, mass)[0, 0, 0]
    assert torch.equal(kept[:keep - recent], torch.arange(keep - recent, dtype=torch.int32, device="cuda"))
    assert torch.equal(kept[keep - recent:], torch.arange(length + 2 - recent, length + 2, dtype=torch.int32, device="cuda"))
    _, v = kv.read([0], [keep - 3], [3])
    assert int((v[0, 0] != 0).sum()) == 0 and int((v[0, 1:] != 0).sum()) > 100
