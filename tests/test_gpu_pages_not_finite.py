"""Values that are no numbers among tokens that rows see, in every kind of workgroup and anywhere in the walk: a row has the infinity or
NaN of the definition, kind by kind, and everything else is what it is without them.  Bounds as in test_gpu_pages.py; weights are
far from vanishing (scores of some tens at most), so an infinity of a token that a row sees is an infinity of the row."""
import math

import pytest
import torch

from tests.test_gpu_pages import fill, make_cache, random_rows, random_tree, sees, shape_of
from tests.test_pages_plan import kinds, plan  # noqa: F401

gpu = pytest.mark.gpu


def definition(q, k, v, seen):
    """(o, S, A) of one client in 64 bits; S of the finite values."""
    rows, nq, dim = q.shape
    group = nq // k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    o, s, a = (torch.zeros(rows, nq, n, dtype=torch.float64) for n in (dim, dim, 1))
    for h in range(k.shape[1]):
        heads = slice(h * group, (h + 1) * group)
        qh = q[:, heads].reshape(rows * group, dim)
        hidden = ~seen.repeat_interleave(group, 0)
        w = torch.softmax((qh @ k[:, h].T / math.sqrt(dim)).masked_fill(hidden, -torch.inf), -1)
        big = (qh.abs() @ k[:, h].abs().nan_to_num(0, posinf=0).T / math.sqrt(dim)).masked_fill(hidden, 0).amax(-1)
        odd = ~torch.isfinite(v[:, h])
        whole = v[:, h].masked_fill(odd, 0)
        oh = w @ whole
        for t in odd.any(-1).nonzero().flatten().tolist():
            who, what = ~hidden[:, t], odd[t].nonzero().flatten()
            oh[who.nonzero(), what] += w[who, t][:, None] * v[t, h, what]
        o[:, heads], s[:, heads], a[:, heads] = oh.view(rows, group, dim), (w @ whole.abs()).view(rows, group, dim), big.view(rows, group, 1)
    return o, s, a


def check(got, want, s, a, dtype):
    got = got.cpu().double()
    for kind in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(kind(got), kind(want)), (kind.__name__, int(kind(got).sum()), int(kind(want).sum()))
    fine = torch.isfinite(want)
    bound = ((2.0 ** -17 if dtype == "f32" else 2.0 ** -8 + 2.0 ** -17) + 2.0 ** -18 * a) * s + 2.0 ** -100
    assert float(((got - want).abs() - bound)[fine].max()) <= 0


def run(heads, dtype, before, rows, tree, spoil, spoil_keys=None):
    nq, nkv, dim = heads
    pg = make_cache(shape_of(*heads, dtype), 1, (before + rows + 15) // 16 + 1)
    k, v = (random_rows(before + rows, nkv, dim, dtype, j) for j in (1, 2))
    spoil(v)
    q = random_rows(rows, nq, dim, dtype, 7)
    if spoil_keys:
        spoil_keys(k, q)
    fill(pg, 0, 0, k, v, before)
    pg.extend([0], [rows], tree)
    pg.append(0, k[before:].cuda(), v[before:].cuda())
    out = pg.attend(0, q.cuda())
    check(out, *definition(q, k, v, sees(before, tree if tree else list(range(-1, rows - 1)))), dtype)


# A wave keeps the blocks of 64 steps at hand (fp32: of 128 tokens): passes of one split whose trees begin in the 64th step and end in
# the 65th.
FAR = [((32, 8, 128), 8064, 256), ((64, 64, 64), 8064, 256)]


@pytest.mark.parametrize("heads,before,rows", FAR)
def test_the_far_passes_walk_more_than_64_steps(plan, heads, before, rows):  # noqa: F811
    assert kinds(plan, heads, "f32", [before], [rows]) == [(2, 1, 0)] and before == 63 * 128 and rows > 128


@gpu
@pytest.mark.parametrize("heads,before,rows", FAR)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_blocks_of_the_64th_step(bad, heads, before, rows):
    def spoil(v):
        for row in (0, 2, 20, 127, 128, 200):
            v[before + row, row % 8, (5 + row) % heads[2]] = bad

    run(heads, "f32", before, rows, random_tree(rows, 3), spoil)


# Passes over texts with infinities: all kinds of workgroups, with and without splits.  In bf16 every walk over one is made twice.
TEXTS = [((8, 2, 64), 300, 1), ((8, 2, 128), 300, 17), ((32, 8, 128), 2048, 64), ((8, 2, 128), 20000, 9), ((32, 8, 64), 500, 300),
         ((32, 8, 128), 9000, 300), ((16, 2, 64), 20000, 33)]


def test_the_texts_reach_every_kind_of_workgroup(plan):  # noqa: F811
    got = {(t, n > 1) for heads, before, rows in TEXTS for t, n, _ in kinds(plan, heads, "bf16", [before], [rows])}
    assert {t for t, _ in got} == {1, 2, 4, 8} and {s for _, s in got} == {True, False}


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,before,rows", TEXTS)
@pytest.mark.parametrize("form", ["chain", "tree"])
def test_infinities_of_the_text(heads, before, rows, dtype, form):
    """Anywhere in the text: infinities of either sign in channels of their own, of both signs and NaN in others."""
    if form == "tree" and rows > 256:
        rows = 256

    def spoil(v):
        tokens, dim = v.shape[0], v.shape[2]
        for i, t in enumerate(range(3, before, max(11, before // 40))):
            v[t, i % v.shape[1], i % 7] = math.inf
            v[t + 1, 0, 8 + i % 7] = -math.inf
            v[t + 2, -1, dim - 1 - i % 3] = math.inf if i % 2 else -math.inf
        v[before // 2, 0, 20] = math.nan
        assert tokens > before

    run(heads, dtype, before, rows, random_tree(rows, rows) if form == "tree" else None, spoil)


@gpu
@pytest.mark.parametrize("heads,before,rows", TEXTS)
def test_one_infinity_wherever_it_lies(heads, before, rows):
    for t in (0, before // 3, before - 33, before - 1):
        for bad in (math.inf, -math.inf):
            run(heads, "bf16", before, rows, None, lambda v: v[t, :, 5].fill_(bad))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,before,rows", TEXTS)
def test_infinities_of_tokens_that_have_no_weight(heads, before, rows, dtype):
    """A key that gives every row a score of -inf: its value's infinity times 0 is no number, and what is finite there does not count."""
    at = {before // 3, before - 20, before + rows // 2}

    def spoil(v):
        for t in at:
            v[t, :, t % 7] = math.inf
        v[before // 2, :, 9] = math.inf  # (of a token that has weight)

    def keys(k, q):
        q[:, :, 3] = q[:, :, 3].abs() + 0.25
        for t in at:
            k[t, :, 3] = -math.inf

    run(heads, dtype, before, rows, None, spoil, keys)


def test_the_long_text_is_walked_in_more_than_64_steps(plan):  # noqa: F811
    assert kinds(plan, (256, 256, 64), "bf16", [17000], [9]) == [(1, 1, 0)] and 17000 > 65 * 256


@gpu
def test_infinities_of_a_walk_of_more_than_64_steps():
    def spoil(v):
        for i, t in enumerate(range(62 * 256 - 40, 65 * 256, 37)):
            v[t, i * 31 % 256, i % 64] = math.inf

    run((256, 256, 64), "bf16", 17000, 9, None, spoil)
