"""Verification on the GPU against its definition in exact fractions, over rows whose sums are anything."""
import numpy as np
import pytest
import torch

import tree_definition
from paper_2402_05099_amd import binding as hb
from test_gpu_ragged import DEV, context, i32, offsets
from test_tree_definition import BY_HAND, ROW, SIBLINGS, draw

pytestmark = pytest.mark.gpu


def run(cases, dtype, mib=0, columns=None):
    """cases: (tokens, parents, target, draft or None, u, u_next) of a sequence each; columns: what lies behind them is 0"""
    off = offsets([len(c[0]) for c in cases])
    T, B, drafts = int(off[-1]), len(cases), cases[0][3] is not None
    cat = lambda i: torch.tensor(np.concatenate([np.asarray(c[i]) for c in cases]))  # noqa: E731
    P, Q = cat(2).to(dtype), cat(3).to(dtype) if drafts else None
    path, kept, nxt = (torch.full((k,), 77, dtype=torch.int32, device=DEV) for k in (T, B, B))
    ctx = context(mib)
    hb.hg_tree_verify(ctx, cat(0).to(torch.int32).to(DEV), cat(1).to(torch.int32).to(DEV), i32(off.tolist()), max(len(c[0]) for c in cases), P.to(DEV), Q.to(DEV) if drafts else None,
                      cat(4).to(DEV), torch.tensor([float(c[5]) for c in cases], device=DEV), path, kept, nxt)
    torch.cuda.synchronize()
    ctx.close()
    for b, c in enumerate(cases):
        at = slice(int(off[b]), int(off[b + 1]))
        want, y = tree_definition.verify(c[0], c[1], P[at, :columns].double().numpy(), Q[at].double().numpy() if drafts else None, c[4], c[5])
        assert path[at].tolist() == want + [-1] * (len(c[0]) - len(want)) and (kept[b].item(), nxt[b].item()) == (len(want), y), b


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [4, 9000, 98304])
def test_the_rule_without_drafts_by_hand(V, dtype):
    P = np.zeros((4, V), dtype=np.float32)
    P[:, :4] = ROW
    run([(SIBLINGS, [-1, 0, 0, 0], P, None, np.array([0, *u], dtype=np.float32), un) for u, _ in BY_HAND for un in (0.0, 0.19, 0.21, 0.9)], dtype, 1, 4)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("drafts", [True, False])
def test_rows_that_sum_to_anything(drafts, dtype):
    r = np.random.default_rng(23)
    for V in (3, 17, 60):
        run([draw(r, int(r.integers(1, 14)), V, drafts) for _ in range(80)], dtype)
