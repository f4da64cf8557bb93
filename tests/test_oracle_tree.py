"""The checker of tree decisions: a chain is the chain's checker, the closed form is the definition, and the accepted text has the
target's law."""
import itertools

import numpy as np
import pytest

from oracle.spec_sampling import spec_accept
from oracle.tree import nested_rule, row_rule, tree_accept

F32 = np.float32


def distribution(rng, vocab, sharp=1.0, zeros=0):
    x = np.exp(sharp * rng.standard_normal(vocab))
    if zeros:
        x[rng.choice(vocab, zeros, replace=False)] = 0
    return (x / x.sum()).astype(F32)


@pytest.mark.parametrize("distinct", [False, True])
@pytest.mark.parametrize("seed", range(8))
def test_a_chain_is_decided_as_a_chain(seed, distinct):
    rng = np.random.default_rng(seed)
    vocab, k = 37, 5
    p = np.stack([distribution(rng, vocab) for _ in range(k + 1)])
    q = np.stack([distribution(rng, vocab) for _ in range(k + 1)])
    d = [int(rng.choice(vocab, p=q[i] / q[i].sum(dtype=np.float64))) for i in range(k)]
    u = rng.integers(0, 1 << 24, k + 1).astype(F32) * F32(2.0 ** -24)
    a, nxt = spec_accept(p, q[:k], d, u)
    path, got = tree_accept(p, q, [0] + d, list(range(-1, k)), [u[k], *u[:k]], distinct)
    assert (path, got) == (list(range(1, a + 1)), nxt)


@pytest.mark.parametrize("distinct", [False, True])
@pytest.mark.parametrize("seed", range(6))
def test_the_closed_form_is_the_definition(seed, distinct):
    """Ratios and residuals of up to four refusals.  Both sides compute in at least 24 bits; a residual that has lost c of its bits to
    cancellation has 24 - c: sums of at least 1e-3 lose 10 at most a step, 2^-24 * 2^10 * 4 steps < 3e-4 relative."""
    rng = np.random.default_rng(100 + seed)
    vocab = 23
    p, q = distribution(rng, vocab, 1.0), distribution(rng, vocab, 1.0)
    tokens = [int(t) for t in rng.choice(vocab, 4, replace=not distinct, p=q / q.sum(dtype=np.float64))]
    ratios, a = row_rule(p, q, tokens, distinct)
    want, residual = nested_rule(p, q, tokens, distinct)
    r = p.astype(np.float64)
    for i, (got, w) in enumerate(zip(ratios, want)):
        refused = [t for t, x in zip(tokens[:i], want) if x < 1]
        if len(refused) < i:
            break  # (a child that is always accepted ends the row)
        assert min(1.0, float(got)) == pytest.approx(w, rel=3e-4, abs=1e-6), i
    else:
        if all(x < 1 for x in want):
            left = np.maximum(0, r - float(a) * q.astype(np.float64))
            assert left / left.sum() == pytest.approx(residual, rel=1e-3, abs=1e-5)


@pytest.mark.parametrize("distinct", [False, True])
@pytest.mark.parametrize("many", [1, 2, 3])
@pytest.mark.parametrize("zeros", [0, 2])
def test_the_first_token_has_the_targets_law(distinct, many, zeros):
    """Over all draws of `many` children: sum of P(draw) (P(child accepted) [its token] + P(all refused) residual) = p.  Every term has
    a relative error of about 2^-20 (fp32 with cancellation at sums above 1e-3), the whole 1e-5."""
    rng = np.random.default_rng(7 + many)
    vocab = 6
    p, q = distribution(rng, vocab, 0.7, zeros), distribution(rng, vocab, 0.7, zeros)
    if distinct and many > vocab - zeros:
        pytest.skip("fewer tokens than draws")
    law = np.zeros(vocab)
    qd = q.astype(np.float64) / q.sum(dtype=np.float64)
    for draw in itertools.product(range(vocab), repeat=many):
        if distinct and len(set(draw)) < many:
            continue
        chance, rest = 1.0, 1.0
        for x in draw:
            chance *= qd[x] / rest if rest > 0 else 0.0
            if distinct:
                rest -= qd[x]
        if chance <= 0:
            continue
        ratios, a = row_rule(p, q, draw, distinct)
        go_on = chance
        for x, r in zip(draw, ratios):
            take = 0.0 if r != r else min(1.0, float(r))
            law[x] += go_on * take
            go_on *= 1 - take
            if go_on <= 0:
                break
        else:
            left = np.maximum(0, p.astype(np.float64) - float(a) * q.astype(np.float64))
            if left.sum() > 0:
                law += go_on * left / left.sum()
    assert law == pytest.approx(p, abs=1e-5)


def test_token_matching_goes_down_the_first_matching_child():
    p = np.eye(5, dtype=F32)[[3, 1, 4, 2, 0]]
    # rows: 0 -> (1: token 2, 2: token 3, 3: token 3), 2 -> (4: token 4)
    assert tree_accept(p, None, [0, 2, 3, 3, 4], [-1, 0, 0, 0, 2], None) == ([2, 4], 0)
    assert tree_accept(p, None, [0, 2, 1, 4, 4], [-1, 0, 0, 0, 2], None) == ([], 3)


def test_special_rows():
    p = np.array([[0.5, 0.5, 0, 0], [0, 0, 1, 0]], F32)
    q = np.array([[0.5, 0.5, 0, 0], [0, 0, 1, 0]], F32)
    # q = p: the first child is always accepted; a child of no mass on both sides never
    assert tree_accept(p, q, [0, 1], [-1, 0], [0.25, 0.999]) == ([1], 2)
    assert tree_accept(p, q, [0, 3], [-1, 0], [0.25, 0.0])[0] == []
    # q(x) = 0 < p(x) is accepted
    q[0] = [0, 0, 0, 1]
    assert tree_accept(p, q, [0, 1], [-1, 0], [0.25, 0.999]) == ([1], 2)
    # nothing left where q covers p: the largest p
    q[0] = p[0]
    path, token = tree_accept(p, q, [0, 2, 2], [-1, 0, 0], [0.9, 0.5, 0.5])
    assert (path, token) == ([], 0)
