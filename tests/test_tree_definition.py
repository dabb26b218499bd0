"""The plain form of verification (tree_plain.py) against its definition in exact fractions, over rows whose sums are anything, and the rule without drafts spelled out on numbers that are exact."""
import numpy as np
import pytest

import tree_definition
import tree_plain as plain


def draw(r, n, V, drafts):
    """A tree, rows that sum to 0.3 .. 1.7 in float32, tokens that are likely in them, random numbers."""
    P, Q = ((r.dirichlet(np.full(V, 0.4), n) * r.uniform(0.3, 1.7, (n, 1))).astype(np.float32) for _ in range(2))
    parents = [-1] + [int(r.integers(max(0, t - 4), t)) for t in range(1, n)]
    tokens = [int(r.choice(V, p=P[max(p, 0)].astype(np.float64) / P[max(p, 0)].astype(np.float64).sum())) for p in parents]
    return tokens, parents, P, Q if drafts else None, r.random(n).astype(np.float32), np.float32(r.random())


# p = (1/2, 1/4, 1/16, 0), which sums to 13/16; siblings 0, 1, 2 of the first token; (u of each) -> what stands, S behind the refusals: 1, 1/2, 1/4, 3/16
ROW, SIBLINGS = [0.5, 0.25, 0.0625, 0.0], [7, 0, 1, 2]
BY_HAND = [((0.49, 0.9, 0.9), 1), ((0.5, 0.49, 0.9), 2), ((0.5, 0.5, 0.24), 3), ((0.5, 0.5, 0.25), 0), ((0.9, 0.9, 0.9), 0)]


@pytest.mark.parametrize("u,stands", BY_HAND)
def test_the_rule_without_drafts_by_hand(u, stands):
    """(u = 0.9 for the second: over the sum of what is left, 5/16, it would stand.)"""
    P = np.array([ROW] * 4, dtype=np.float32)
    for verify in (plain.verify, tree_definition.verify):
        path, _ = verify(SIBLINGS, [-1, 0, 0, 0], P, None, np.array([0, *u], dtype=np.float32), 0.0)
        assert path == ([0, stands] if stands else [0])


@pytest.mark.parametrize("drafts", [True, False])
def test_the_plain_form_is_the_definition(drafts):
    r, kept = np.random.default_rng(5), 0
    for _ in range(300):
        case = draw(r, int(r.integers(1, 14)), int(r.integers(1, 12)), drafts)
        got = plain.verify(*case)
        assert got == tree_definition.verify(*case)
        kept += len(got[0]) - 1
    assert kept > 150
