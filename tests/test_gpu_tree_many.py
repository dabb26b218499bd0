"""Masks of more sequences than one launch of 512 threads to each 64 tokens of each has room for."""
import numpy as np
import pytest
import torch

import tree_plain as plain
from paper_2402_05099_amd import binding as hb
from test_gpu_ragged import DEV, context, i32
from test_gpu_trees import random_parents

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("most", [64, 65, 1024])
def test_masks_of_half_a_million_sequences(most):
    B, per_launch, r = 530001, 0xffffffff // (512 * 16), np.random.default_rng(most)
    trees = {0: 5, 1: 70, per_launch - 1: 64, per_launch: 130, per_launch + 1: 1, 262143: 200, B - 1: 90}
    counts = np.zeros(B, dtype=np.int64)
    for b, n in trees.items():
        counts[b] = n
    off = np.concatenate([[0], np.cumsum(counts)])
    T = int(off[-1])
    words = -(-min(most, T) // 32)
    parents, want, deep = np.full(T, -1), np.full((T, words), 77, dtype=np.int32), np.full(T, 77)
    for b, n in trees.items():
        a, take = int(off[b]), min(n, most)
        up = random_parents(r, n, 4)
        parents[a:a + n] = up
        m = plain.follows(up)[:take, :take]
        want[a:a + take] = plain.words(m, words)
        deep[a:a + take] = m.sum(1) - 1
    got, d = torch.full((T, words), 77, dtype=torch.int32, device=DEV), torch.full((T,), 77, dtype=torch.int32, device=DEV)
    ctx = context()
    hb.hg_tree_masks(ctx, i32(parents.tolist()), torch.tensor(off, dtype=torch.int32, device=DEV), most, got, d)
    torch.cuda.synchronize()
    ctx.close()
    assert np.array_equal(got.cpu().numpy(), want) and d.tolist() == deep.tolist()
