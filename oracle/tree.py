"""Decision on a tree of drafts (checker).

The speculative-sampling rule of oracle/spec_sampling.py for several drafts at a place: children of a row are tried in order against
what the target still wants.  With r_0 = p and s_i the draft distribution that child i was drawn from (q, or without the refused
drafts and renormalised), child i is accepted with probability min(1, r_i(x) / s_i(x)), and a refusal leaves r_{i+1} = max(0, r_i - s_i)
normalised.  `nested_rule` is that definition in 64 bits.  `tree_accept` is the form that the library fixes to the last bit: r_i is
max(0, p - a_i q) / T_i with a_{i+1} = a_i + T_i / S_i, sums of whole numbers floor(2^40 w), fp32 numbers where it says so.
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import numpy as np

from oracle.spec_sampling import draw_index

F32 = np.float32
ONE = F32(1)


def nested_rule(p, q, tokens: Sequence[int], distinct: bool):
    """(acceptance probabilities of the children, residual behind the last), by the definition in 64 bits."""
    r, s = np.asarray(p, np.float64) / np.sum(p, dtype=np.float64), np.asarray(q, np.float64) / np.sum(q, dtype=np.float64)
    out = []
    for x in tokens:
        out.append(min(1.0, r[x] / s[x]) if s[x] > 0 else (1.0 if r[x] > 0 else 0.0))
        r = np.maximum(0.0, r - s)
        r = r / r.sum() if r.sum() > 0 else r
        if distinct:
            s = s.copy()
            s[x] = 0.0
            s = s / s.sum() if s.sum() > 0 else s
    return out, r


def left_of(p: np.ndarray, q: np.ndarray, a) -> np.ndarray:
    """max(0, p - a q) in fp32, the difference rounded once.  (Products of fp32 numbers are exact in fp64, their difference from p mostly is: where
    it needs more than 53 bits, and what is cut off decides a tie of the rounding to fp32, one operation on fp32 numbers is off by an ulp,
    about once in 2^28.)"""
    return np.maximum(F32(0), (p.astype(np.float64) - np.float64(a) * q.astype(np.float64)).astype(F32))


def row_rule(p: np.ndarray, q: np.ndarray, tokens: Sequence[int], distinct: bool):
    """Per child the ratio that its uniform is compared with; behind the last the a of what is left."""
    a, b, mass, ratios = F32(0), ONE, 1.0, []
    for i, x in enumerate(tokens):
        if i:
            total = int(np.floor(left_of(p, q, a).astype(np.float64) * 2.0 ** 40).astype(np.uint64).sum())
            b = F32(total * 2.0 ** -40 / mass)
        with np.errstate(divide="ignore", invalid="ignore"):
            ratios.append(left_of(p[x:x + 1], q[x:x + 1], a)[0] / (b * q[x]))
        a = F32(a + b)
        if distinct:
            mass = max(mass - float(q[x]), 2.0 ** -24)
    return ratios, a


def tree_accept(p: np.ndarray, q: Optional[np.ndarray], tokens: Sequence[int], parents: Sequence[int], u, distinct: bool = False):
    """(accepted rows, next token) of one client's tree; rows 0 .. n - 1, row 0 the pending token's."""
    n, at, path = len(tokens), 0, []  # type: int, int, List[int]
    while True:
        children = [c for c in range(1, n) if parents[c] == at]
        taken = None
        if q is None:
            best = int(np.argmax(p[at]))
            taken = next((c for c in children if tokens[c] == best), None)
        else:
            ratios, a = row_rule(p[at], q[at], [tokens[c] for c in children], distinct)
            taken = next((c for c, r in zip(children, ratios) if r == r and F32(u[c]) < min(ONE, r)), None)  # (0 / 0 refuses)
        if taken is None:
            break
        path.append(taken)
        at = taken
    if q is None:
        return path, int(np.argmax(p[at]))
    return path, draw_index(left_of(p[at], q[at], a) if children else p[at].astype(F32), u[0], p[at])
