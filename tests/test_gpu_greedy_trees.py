"""Greedy steps over drafted trees say what the model says token by token, in 64 bits, but for the roundings of the attention: the toy of examples/drafted_trees.py with an attention that decides as
much as the last token does."""
import os
import sys

import pytest

from greedy_check import Exact, worst

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("heads,dim,branches,codes", [((8, 2), 128, [3, 2, 2], False), ((16, 2), 64, [4, 3], True), ((4, 4), 64, [1, 1, 1, 1], False), ((8, 1), 128, [2, 2, 2, 2, 2], True),
                                                      ((16, 2), 128, [6, 6], False)])
def test_greedy_texts_are_the_models(heads, dim, branches, codes):
    from test_gpu_drafted_trees import run
    steps, B = 10, 5
    model, server, texts = run(heads, dim, branches, codes, True, steps=steps, B=B, attends=6.0)
    assert sum(len(t) - 1 for t in texts) > 1.15 * steps * B      # drafts have stood
    exact = Exact(model, codes)
    far = [worst(exact, text) for text in texts]
    assert max(far) <= 1, far
