"""Plain forms of the calls of a decode step over drafted trees, in 64 bits and by their definitions: what the GPU tests and the example compare with.  Loops over sequences and
tokens, no code of the library."""
import math

import numpy as np
import torch


def parents_of(t, parents):
    """parents[t] where it is a parent, else None"""
    p = int(parents[t])
    return p if 0 <= p < t else None


def follows(parents):
    """[n, n] truth values: j is t or one of its ancestors"""
    n = len(parents)
    m = np.zeros((n, n), dtype=bool)
    for t in range(n):
        p = parents_of(t, parents)
        if p is not None:
            m[t] = m[p]
        m[t, t] = True
    return m


def words(m, count):
    """truth values [n, k] as int32 words [n, count]"""
    out = np.zeros((m.shape[0], count), dtype=np.uint32)
    for j in range(min(m.shape[1], 32 * count)):
        out[:, j // 32] |= m[:, j].astype(np.uint32) << np.uint32(j % 32)
    return out.view(np.int32)


def attention(Q, q_off, sees, keys, values, lens, scale=None, max_new=None):
    """O and LSE (float64) of packed tokens; sees[b]: [n, n] truth values; keys[b], values[b]: float64 [len_b, Hkv, D].  Tokens that are not computed are NaN."""
    T, Hq, D = Q.shape
    O, L = torch.full((T, Hq, D), math.nan, dtype=torch.float64), torch.full((T, Hq), math.nan, dtype=torch.float64)
    scale = 1 / math.sqrt(D) if scale is None else scale
    Q = Q.detach().cpu().double()
    for b in range(len(q_off) - 1):
        q0, n = int(q_off[b]), int(q_off[b + 1]) - int(q_off[b])
        take = n if max_new is None else min(n, max_new)
        if take == 0:
            continue
        rows = int(lens[b])
        k, v = keys[b].double()[:rows], values[b].double()[:rows]
        G = Hq // k.shape[1]
        for t in range(take):
            which = [j for j in range(rows) if j < rows - n or sees[b][t, j - (rows - n)]]
            if not which:
                O[q0 + t], L[q0 + t] = 0.0, -math.inf
                continue
            kk, vv = k[which].repeat_interleave(G, 1), v[which].repeat_interleave(G, 1)
            s = (Q[q0 + t][None] * kk).sum(2) * scale      # [keys, Hq]
            L[q0 + t] = torch.logsumexp(s, 0)
            O[q0 + t] = (torch.exp(s - L[q0 + t])[:, :, None] * vv).sum(0)
    return O, L


def counted(x):
    x = np.asarray(x, dtype=np.float64)
    return np.where(np.isfinite(x) & (x > 0), x, 0.0)


def verify(tokens, parents, target, draft, u, u_next):
    """(path, next token) of one sequence, as the definition has it: what is left after a refusal is max(0, p - q) (or p without the token) over its sum.  target: [n, V], or n tokens."""
    n = len(tokens)
    if n == 0:
        return [], -1
    cur, path = 0, [0]
    left = None if np.ndim(target) == 1 else counted(target[0])
    whole = 1.0      # what `left` counts as
    for t in range(1, n):
        if parents_of(t, parents) != cur:
            continue
        x = int(tokens[t])
        if np.ndim(target) == 1:
            if x == int(target[cur]):
                cur = t
                path.append(t)
            continue
        inside = 0 <= x < len(left)
        p = left[x] / whole if inside and whole != 0 else 0.0
        q = (counted(draft[cur])[x] if inside else 0.0) if draft is not None else 1.0
        if (draft is not None or whole > 0) and float(u[t]) * q < p or (draft is None and whole <= 0 and inside and left[x] > 0):
            cur = t
            path.append(t)
            left, whole = counted(target[cur]), 1.0
        elif draft is not None:
            left = np.maximum(0.0, (left / whole if whole > 0 else left) - counted(draft[cur]))
            whole = left.sum()
        else:
            whole -= left[x] if inside else 0.0
            left = left.copy()
            if inside:
                left[x] = 0.0
    if np.ndim(target) == 1:
        return path, int(target[cur])
    w = left if left.sum() > 0 else counted(target[cur])
    if not w.sum() > 0:
        return path, -1
    passed = np.nonzero((np.cumsum(w) > float(u_next) * w.sum()) & (w > 0))[0]
    return path, int(passed[0]) if len(passed) else int(np.nonzero(w > 0)[0][-1])


def keep(pools, table, ps, q_off, path, accepted, lengths, max_new):
    """(pools, lengths) after the move, row by row.  pools: arrays [pool rows, ...]"""
    pools, table, grown = [np.array(p) for p in pools], np.asarray(table), []
    for b in range(len(q_off) - 1):
        n = int(q_off[b + 1]) - int(q_off[b])
        a, before = min(max(int(accepted[b]), 0), n, max_new), max(int(lengths[b]), 0) - n

        def place(j):
            if j < 0 or j // ps >= table.shape[1]:
                return None
            page = int(table[b, j // ps])
            return page * ps + j % ps if 0 <= page < len(pools[0]) // ps else None

        for i in range(a):
            t = int(path[int(q_off[b]) + i])
            if not i < t < n:
                continue
            src, dst = place(before + t), place(before + i)
            if src is not None and dst is not None:
                for p in pools:
                    p[dst] = p[src]
        grown.append(max(before + a, 0))
    return pools, grown
