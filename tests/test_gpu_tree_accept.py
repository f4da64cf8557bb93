"""The decision on trees of drafts against its checker, to the last bit: small and large vocabularies, trees of one row to 256, rows of
many children, drafts that come twice, rows that leave nothing, many clients in a call, wider matrices, token matching, recorded
calls."""
import numpy as np
import pytest
import torch

from oracle.tree import tree_accept as checker
from paper_2605_13319_amd import nav

gpu = pytest.mark.gpu


def make_tree(rng, rows, children):
    parents, have = [-1], [0]
    for i in range(1, rows):
        j = int(rng.choice([x for x in range(i) if have[x] < children]))
        parents.append(j)
        have[j] += 1
        have.append(0)
    return parents


def make_case(seed, rows, vocab, children, distinct, noise=0.7, zeros=0.0):
    """p, q [rows][vocab], tokens, parents, uniforms of one client."""
    rng = np.random.default_rng(seed)
    z = 3 * rng.standard_normal((rows, vocab))
    y = z + noise * rng.standard_normal((rows, vocab))
    p, q = (np.exp(x - x.max(-1, keepdims=True)) for x in (z, y))
    if zeros:
        p *= rng.random((rows, vocab)) >= zeros
        q *= rng.random((rows, vocab)) >= zeros
        p[:, 0] += 1e-3
        q[:, 1] += 1e-3
    p, q = ((x / x.sum(-1, keepdims=True)).astype(np.float32) for x in (p, q))
    parents = make_tree(rng, rows, children)
    tokens = [0] * rows
    for r in range(rows):
        mine = [c for c in range(1, rows) if parents[c] == r]
        w = q[r].astype(np.float64)
        w /= w.sum()
        many = len(mine)
        got = rng.choice(vocab, many, replace=not distinct or many > np.count_nonzero(w), p=w) if many else []
        for c, x in zip(mine, got):
            tokens[c] = int(x)
    u = (rng.integers(0, 1 << 24, rows) * 2.0 ** -24).astype(np.float32)
    return p, q, tokens, parents, u


def decide(cases, distinct=False, match=False, **kw):
    p = torch.from_numpy(np.concatenate([c[0] for c in cases])).cuda()
    q = None if match else torch.from_numpy(np.concatenate([c[1] for c in cases])).cuda()
    flat = lambda i: [x for c in cases for x in c[i]]
    rows = [len(c[2]) for c in cases]
    u = None if match else np.concatenate([c[4] for c in cases])
    got = nav.tree_accept(p, q, flat(2), flat(3), u, rows=rows, distinct=distinct, **kw)
    torch.cuda.synchronize()
    return got.cpu().tolist()


def expect(cases, distinct=False, match=False, width=None):
    width = width or max(len(c[2]) for c in cases) + 1
    out = []
    for p, q, tokens, parents, u in cases:
        path, token = checker(p, None if match else q, tokens, parents, u, distinct)
        out.append([len(path), token] + path + [-1] * (width - 2 - len(path)))
    return out


@gpu
@pytest.mark.parametrize("distinct", [False, True])
@pytest.mark.parametrize("vocab", [1, 2, 5, 63, 64, 65, 1000, 32000])
def test_small_trees(vocab, distinct):
    deep = 0
    for seed in range(12):
        rows = 1 + seed * 2
        cases = [make_case(1000 * vocab + seed, rows, vocab, 1 + seed % 4, distinct and vocab > 4)]
        want = expect(cases, distinct)
        assert decide(cases, distinct) == want, seed
        deep = max(deep, want[0][0])
    assert deep > 0


@gpu
@pytest.mark.parametrize("distinct", [False, True])
def test_rows_of_many_children(distinct):
    """Children that are refused one after the other: drafts of a distribution far from the target's."""
    for seed, (rows, children, vocab) in enumerate([(10, 9, 300), (40, 39, 2000), (256, 255, 5000), (256, 20, 700), (100, 30, 50)]):
        case = make_case(seed, rows, vocab, children, distinct, noise=4.0)
        want = expect([case], distinct)
        assert decide([case], distinct) == want, seed
        high = (*case[:4], np.full(rows, 0.9999, np.float32))  # (all that may be refused are)
        assert decide([high], distinct) == expect([high], distinct), seed


@gpu
@pytest.mark.parametrize("distinct", [False, True])
def test_the_largest_vocabularies(distinct):
    for seed, (vocab, rows) in enumerate([(128256, 33), (200001, 7), (131073, 12)]):
        case = make_case(50 + seed, rows, vocab, 3, distinct)
        assert decide([case], distinct) == expect([case], distinct)


@gpu
@pytest.mark.parametrize("distinct", [False, True])
def test_rows_without_mass(distinct):
    """Tokens that either side gives nothing, drafts that come twice, targets that the draft distribution covers."""
    for seed in range(10):
        case = make_case(200 + seed, 30, 40, 6, False, zeros=0.6)
        assert decide([case], distinct) == expect([case], distinct), seed
        p, q, tokens, parents, u = make_case(300 + seed, 20, 30, 5, False)
        same = (p, p.copy(), [5] * 20, parents, u)
        assert decide([same], distinct) == expect([same], distinct), seed
        eye = np.eye(30, dtype=np.float32)[np.arange(20) % 30]
        sure = (eye, q, tokens, parents, u)
        assert decide([sure], distinct) == expect([sure], distinct), seed
        sure = (eye, eye[::-1].copy(), tokens, parents, np.full(20, 1 - 2.0 ** -24, np.float32))
        assert decide([sure], distinct) == expect([sure], distinct), seed


@gpu
def test_distributions_that_are_no_numbers_end_the_walk_in_bounds():
    p, q, tokens, parents, u = make_case(1, 12, 500, 3, False)
    for bad in (np.nan, np.inf):
        for x in (p, q):
            x = x.copy()
            x[:, 100:140] = bad
            for args in ((x, q), (p, x), (x, x)):
                got = decide([(*args, tokens, parents, u)])[0]
                assert 0 <= got[0] < 12 and 0 <= got[1] < 500


@gpu
@pytest.mark.parametrize("distinct,match", [(False, False), (True, False), (False, True)])
def test_many_clients(distinct, match):
    """More clients and rows than a launch takes, with one workspace, twice."""
    rng = np.random.default_rng(5)
    cases = [make_case(400 + i, int(n), 333, 4, distinct) for i, n in enumerate(rng.integers(1, 60, 37))] + [make_case(9, 256, 333, 9, distinct)]
    if match:
        for c in cases:  # some drafts are the target's own
            for i in range(1, len(c[2])):
                if rng.random() < 0.6:
                    c[2][i] = int(c[0][c[3][i]].argmax())
    work = nav.tree_workspace(len(cases), sum(len(c[2]) for c in cases))
    result = torch.full((len(cases), 300), 5, dtype=torch.int32, device="cuda")
    want = expect(cases, distinct, match, 300)
    assert max(w[0] for w in want) > 2
    for _ in range(2):
        assert decide(cases, distinct, match, workspace=work, result=result) == want
    for c, w in zip(cases, want):  # what a client gets does not depend on the others
        assert decide([c], distinct, match, workspace=work)[0] == w[:len(c[2]) + 1]


@gpu
def test_equal_largest_probabilities_are_the_lowest_index():
    p = torch.full((4, 1000), 0.001, device="cuda")
    p[1, 700], p[1, 900] = 0.5, 0.5
    got = nav.tree_accept(p, None, [0, 0, 5, 700], [-1, 0, 0, 1], None)
    assert got.cpu().tolist() == [[2, 0, 1, 3, -1]]


@gpu
def test_rows_of_wider_matrices():
    p, q, tokens, parents, u = make_case(77, 25, 999, 3, True)
    wide = torch.full((25, 2100), float("nan"), device="cuda")
    wide[:, 3:1002], wide[:, 1050:2049] = torch.from_numpy(p).cuda(), torch.from_numpy(q).cuda()
    got = nav.tree_accept(wide[:, 3:1002], wide[:, 1050:2049], tokens, parents, u.tolist(), distinct=True)
    assert got.cpu().tolist() == expect([(p, q, tokens, parents, u)], True)


@gpu
def test_a_chain_is_what_the_chains_decision_gives():
    for seed in range(6):
        k, vocab = 9, 4096
        p, q, tokens, _, u = make_case(600 + seed, k + 1, vocab, 1, False)
        parents = list(range(-1, k))
        rng = np.random.default_rng(seed)
        for i in range(1, k + 1):
            tokens[i] = int(rng.choice(vocab, p=q[i - 1] / q[i - 1].sum(dtype=np.float64)))
        pd, qd = torch.from_numpy(p).cuda(), torch.from_numpy(q).cuda()
        a, token = nav.spec_accept(pd, qd[:k].contiguous(), tokens[1:], [*u[1:].tolist(), float(u[0])])
        got = nav.tree_accept(pd, qd, tokens, parents, u).cpu().tolist()[0]
        assert got[:2] == [a, token] and got[2:2 + a] == list(range(1, a + 1))


@gpu
def test_a_recorded_decision():
    """Recorded with its drafts, replayed on other distributions, eager decisions on another workspace between."""
    p, q, tokens, parents, u = make_case(88, 40, 3001, 4, True)
    pd, qd = torch.from_numpy(p).cuda(), torch.from_numpy(q).cuda()
    work, other = nav.tree_workspace(1, 40), nav.tree_workspace(1, 40)
    result = torch.zeros(1, 41, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nav.tree_accept(pd, qd, tokens, parents, u, distinct=True, result=result, workspace=work)
    for seed in range(5):
        p2, q2, *_ = make_case(900 + seed, 40, 3001, 4, True)
        pd.copy_(torch.from_numpy(p2))
        qd.copy_(torch.from_numpy(q2))
        graph.replay()
        torch.cuda.synchronize()
        want = expect([(p2, q2, tokens, parents, u)], True)
        assert result.cpu().tolist() == want
        assert nav.tree_accept(pd, qd, tokens, parents, u, distinct=True, workspace=other).cpu().tolist() == want


@gpu
def test_rows_that_share_memory_are_refused():
    one = torch.full((1, 50), 0.02, device="cuda")
    p = one.expand(3, 50).contiguous()
    shared = torch.rand(200, device="cuda").as_strided((3, 50), (40, 1))
    for bad in (one.expand(3, 50), shared):
        with pytest.raises(ValueError, match="apart"):
            nav.tree_accept(bad, None, [0, 1, 2], [-1, 0, 0], None)
        with pytest.raises(ValueError, match="apart"):
            nav.tree_accept(p, bad, [0, 1, 2], [-1, 0, 0], [0.5] * 3)
    assert nav.tree_accept(one.as_strided((1, 50), (1, 1)), None, [0], [-1], None).tolist() == [[0, 0]]
