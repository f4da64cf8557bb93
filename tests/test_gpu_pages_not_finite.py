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
        big = (qh.abs() @ k[:, h].abs().T / math.sqrt(dim)).masked_fill(hidden, 0).amax(-1)
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


def run(heads, dtype, before, rows, tree, spoil):
    nq, nkv, dim = heads
    pg = make_cache(shape_of(*heads, dtype), 1, (before + rows + 15) // 16 + 1)
    k, v = (random_rows(before + rows, nkv, dim, dtype, j) for j in (1, 2))
    spoil(v)
    fill(pg, 0, 0, k, v, before)
    pg.extend([0], [rows], tree)
    pg.append(0, k[before:].cuda(), v[before:].cuda())
    q = random_rows(rows, nq, dim, dtype, 7)
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
