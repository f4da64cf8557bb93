"""The decision on trees over vocabularies that several workgroups share, against its oracle to the last bit: many clients in a call, rows of
many children, equal maxima in different parts of a row, distributions that are no numbers, calls of different sizes on one
workspace."""
import numpy as np
import pytest
import torch

from paper_2605_13319_amd import nav
from tests.test_gpu_tree_accept import decide, expect, make_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [8193, 20021])
@pytest.mark.parametrize("distinct,match", [(False, False), (True, False), (False, True)])
def test_many_clients(vocab, distinct, match):
    rng = np.random.default_rng(vocab)
    sizes = [1, 40, 2, 17, 64, 1, 9, 33, 5, 1, 1, 30, 12, 3, 8, 21, 6, 50, 2, 11]  # (more clients, and more rows, than a launch takes)
    cases = [make_case(vocab + i, n, vocab, 1 + i % 5, distinct, noise=1.5) for i, n in enumerate(sizes)]
    if match:
        for c in cases:  # some drafts are the target's own
            for i in range(1, len(c[2])):
                if rng.random() < 0.6:
                    c[2][i] = int(c[0][c[3][i]].argmax())
    else:
        for c in cases[::3]:
            c[4][1:] = 0.9999  # (all that may be refused are: every launch has something to do)
    work = nav.tree_workspace(len(cases), sum(sizes))
    result = torch.full((len(cases), 70), 5, dtype=torch.int32, device="cuda")
    want = expect(cases, distinct, match, 70)
    assert max(w[0] for w in want) > 1 and min(w[0] for w in want) == 0
    for _ in range(2):
        assert decide(cases, distinct, match, workspace=work, result=result) == want
    for c, w in zip(cases[:6], want):  # what a client gets does not depend on the others
        assert decide([c], distinct, match, workspace=work)[0] == w[:len(c[2]) + 1]


@pytest.mark.parametrize("distinct", [False, True])
@pytest.mark.parametrize("rows,children,vocab", [(10, 9, 20021), (30, 12, 9001), (256, 255, 8200), (120, 40, 33000)])
def test_rows_of_many_children(rows, children, vocab, distinct):
    case = make_case(rows + vocab, rows, vocab, children, distinct, noise=4.0)
    assert decide([case], distinct) == expect([case], distinct)
    high = (*case[:4], np.full(rows, 0.9999, np.float32))
    assert decide([high], distinct) == expect([high], distinct)
    u = case[4].copy()
    first = [c for c in range(1, rows) if case[3][c] == 0]
    u[first[:-1]] = 1 - 2.0 ** -24  # the last child of the first row, behind all others' sums
    last = (*case[:4], u)
    assert decide([last, case], distinct) == expect([last, case], distinct)


def test_equal_largest_probabilities_in_different_parts_are_the_lowest_index():
    for vocab, places in ((30000, (5, 29999)), (30000, (2999, 3000, 20000)), (131073, (131072, 65000)), (8193, (8192, 4096))):
        p = torch.full((4, vocab), 1e-6, device="cuda")
        p[1, list(places)], p[0, 7], p[2, vocab - 1] = 0.4, 0.5, 0.5
        low = min(places)
        got = nav.tree_accept(p, None, [0, 7, max(places), low], [-1, 0, 1, 1], None)
        assert got.cpu().tolist() == [[2, 0, 1, 3, -1]]
        got = nav.tree_accept(p, None, [0, 7, max(places), vocab - 1], [-1, 0, 1, 2], None)
        assert got.cpu().tolist() == [[1, low, 1, -1, -1]]


@pytest.mark.parametrize("distinct", [False, True])
def test_rows_without_mass(distinct):
    """Tokens that either side gives nothing, drafts that come twice, targets that the draft distribution covers."""
    vocab = 10001
    for seed in range(3):
        case = make_case(200 + seed, 24, vocab, 5, False, zeros=0.9)
        assert decide([case], distinct) == expect([case], distinct), seed
        p, q, tokens, parents, u = make_case(300 + seed, 20, vocab, 5, False)
        same = (p, p.copy(), [9000] * 20, parents, u)
        assert decide([same], distinct) == expect([same], distinct), seed
        eye = np.zeros((20, vocab), np.float32)
        eye[np.arange(20), (np.arange(20) * 521) % vocab] = 1
        for d in (q, eye[::-1].copy()):
            sure = (eye, d, tokens, parents, np.full(20, 1 - 2.0 ** -24, np.float32))
            assert decide([sure], distinct) == expect([sure], distinct), seed


def test_distributions_that_are_no_numbers_end_the_walk_in_bounds():
    vocab = 20021
    p, q, tokens, parents, u = make_case(1, 12, vocab, 3, False)
    work = nav.tree_workspace(1, 12)
    for bad in (np.nan, np.inf):
        for x in (p, q):
            x = x.copy()
            x[:, 2000:15000] = bad
            for args in ((x, q), (p, x), (x, x)):
                for match in (False, True):
                    got = decide([(*args, tokens, parents, u)], match=match, workspace=work)[0]
                    assert 0 <= got[0] < 12 and 0 <= got[1] < vocab
    fine = [(p, q, tokens, parents, u)]
    assert decide(fine, workspace=work) == expect(fine)  # (and leave the workspace as the next call needs it)


def test_calls_of_all_sizes_on_one_workspace():
    work = nav.tree_workspace(1, 1)
    for seed, (vocab, rows, match) in enumerate([(128256, 20, False), (50, 30, False), (9000, 9, False), (33000, 64, True), (8192, 40, False), (40000, 3, False),
                                                 (1, 1, True), (200001, 5, False), (20021, 33, False)]):
        case = [make_case(700 + seed, rows, vocab, 4, False, noise=2.0)]
        assert decide(case, match=match, workspace=work) == expect(case, match=match), vocab
