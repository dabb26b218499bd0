"""Verification of a tree of drafted tokens by its definition in exact fractions (no rounding, no code of the library or of tree_plain.py), for rows that sum to anything."""
import math
from fractions import Fraction


def exact(x):
    x = float(x)
    return Fraction(x) if math.isfinite(x) and x > 0 else Fraction(0)


def verify(tokens, parents, target, draft, u, u_next):
    """(tokens that stand, next token).  With draft: u q(x) < p_k(x), and p_k+1 = max(0, p_k - q) over its sum.  Without: u S_k < p(x), S_0 = 1, S_k+1 = S_k - p(x), and the refused x has nothing
    left."""
    path, cur = [0], 0
    row = [exact(x) for x in target[0]]
    left, S = row, Fraction(1)
    for t in range(1, len(tokens)):
        if int(parents[t]) != cur:      # (a parent at or behind t is none, and no such t has `cur` for one)
            continue
        x, ut = int(tokens[t]), Fraction(float(u[t]))
        p = left[x] if 0 <= x < len(left) else Fraction(0)
        if draft is None:
            stands = p > 0 and ut * S < p
        else:
            q = [exact(y) for y in draft[cur]]
            stands = ut * (q[x] if 0 <= x < len(q) else Fraction(0)) < p
        if stands:
            path.append(t)
            cur, row = t, [exact(y) for y in target[t]]
            left, S = row, Fraction(1)
        elif draft is None:
            left = [Fraction(0) if y == x else v for y, v in enumerate(left)]
            S -= p
        else:
            left = [max(Fraction(0), v - w) for v, w in zip(left, q)]
            whole = sum(left)
            left = [v / whole for v in left] if whole > 0 else left
    w = left if sum(left) > 0 else row
    whole, run = sum(w), Fraction(0)
    if whole == 0:
        return path, -1
    for y, v in enumerate(w):
        run += v
        if v > 0 and run > Fraction(float(u_next)) * whole:
            return path, y
    return path, max(y for y, v in enumerate(w) if v > 0)
