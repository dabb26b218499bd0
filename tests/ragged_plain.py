"""Plain forms of the calls between a prompt and its first decode step, in 64 bits and by their definitions: what the GPU tests and the example
compare with.  Loops over sequences and tokens, no code of the library."""
import math

import numpy as np
import torch


def attention(Q, q_off, keys, values, lens, scale=None, max_new=None):
    """O and LSE (float64) of packed tokens; keys[b], values[b]: float64 [len_b, Hkv, D].  Tokens that are not computed are NaN."""
    T, Hq, D = Q.shape
    O, L = torch.full((T, Hq, D), math.nan, dtype=torch.float64), torch.full((T, Hq), math.nan, dtype=torch.float64)
    scale = 1 / math.sqrt(D) if scale is None else scale
    Q = Q.detach().cpu().double()
    for b in range(len(q_off) - 1):
        q0, q1 = int(q_off[b]), int(q_off[b + 1])
        n = q1 - q0
        take = n if max_new is None else min(n, max_new)
        if take == 0:
            continue
        k, v, rows = keys[b].double(), values[b].double(), int(lens[b])
        G = Hq // k.shape[1]
        kk, vv = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
        S = torch.einsum("thd,jhd->htj", Q[q0:q0 + take], kk[:rows]) * scale
        seen = rows - (n - 1 - torch.arange(take))
        S.masked_fill_(torch.arange(rows)[None, None, :] >= seen[None, :, None], -math.inf)
        lse = torch.logsumexp(S, 2) if rows else torch.full((Hq, take), -math.inf, dtype=torch.float64)
        W = torch.exp(S - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, :, None])
        O[q0:q0 + take] = torch.einsum("htj,jhd->thd", W, vv[:rows])
        L[q0:q0 + take] = lse.T
    return O, L


def page_slots(lengths, counts, free, ps, table, rows):
    """(q_off, slots, new_lengths, pages_used, table) by walking sequence after sequence, token after token"""
    table = np.array(table)
    cap = table.shape[1] * ps
    q_off, slots, new, taken = [0], [], [], 0
    for b, (x, n) in enumerate(zip(lengths, counts)):
        x, n = max(int(x), 0), max(int(n), 0)
        placed = x
        for j in range(x, x + n):
            if j >= cap:
                slots.append(-1)
                continue
            if j % ps == 0:
                table[b, j // ps] = free[taken] if taken < len(free) else -1
                taken += 1
            page = table[b, j // ps]
            slots.append(int(page) * ps + j % ps if page >= 0 else -1)
            placed += page >= 0
        q_off.append(q_off[-1] + n)
        new.append(placed)
    slots = (slots + [-1] * rows)[:rows]
    return np.array(q_off), np.array(slots), np.array(new), taken, table
