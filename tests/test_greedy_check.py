"""The check of greedy texts (greedy_check.py) takes what rounding does and rejects attention that sees a row too few or too many."""
import os
import sys

import pytest
import torch

from greedy_check import Exact, worst, wrong_texts

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("heads,dim,codes", [((8, 2), 128, False), ((16, 2), 64, True)])
@pytest.mark.parametrize("what", ["rounded", "parent", "siblings", "none"])
def test_what_the_check_takes_and_rejects(what, heads, dim, codes):
    from drafted_trees import Toy
    exact = Exact(Toy(2, heads, dim, 60, 64, attends=6.0, device="cpu"), codes)
    far = [worst(exact, text) for text in wrong_texts(exact, what)]
    if what == "rounded":
        assert max(far) <= 1
    else:
        assert min(far) > 3, far      # every one of the texts, and by far
