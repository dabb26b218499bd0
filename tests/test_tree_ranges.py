"""Whether the attention of drafted trees splits the keys of its tiles, checked without a GPU: a few large trees behind long contexts among requests of few tokens are split wherever the same
batch of chunks is, whatever the number of requests and heads."""
import random

import pytest

from paper_2402_05099_amd import binding as hb
from test_tree_plans import look

WS = 1 << 40


def plans(seqs, heads, D, codes=False, max_len=None, ws=WS):
    """seqs: (rows in the cache, new tokens).  The plans of the tree call and of the chunk call on the same batch"""
    counts = [n for _, n in seqs]
    size = (sum(counts), max_len or max(x for x, _ in seqs), len(seqs), *heads, D, max(counts), codes, ws)
    return look(*size), hb.hg_debug_ragged_plan(*size, tree=False)


def one_large(B, n=64, keys=65536, others=2):
    return [(keys, n)] + [(300 + 7 * b % 600, others) for b in range(B - 1)]


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads,B", [((40, 40), 20), ((40, 40), 64), ((40, 40), 65), ((32, 32), 32), ((16, 16), 64), ((64, 16), 60), ((32, 8), 90), ((32, 8), 96), ((32, 8), 100), ((32, 8), 255),
                                     ((32, 8), 256), ((32, 8), 257), ((32, 32), 200), ((8, 1), 256), ((40, 40), 256)])
def test_a_large_tree_among_single_requests_is_split(heads, B, D, codes):
    """A tile of 65536 keys is 2048 stages of 0.6 us, 1.2 ms, where all of its bytes and those of the others are 0.1 to 0.4."""
    tree, chunk = plans(one_large(B), heads, D, codes)
    assert tree["tiles"] and tree["tile_nsplit"] >= chunk["tile_nsplit"] > 1


@pytest.mark.parametrize("edge", [767, 768, 769])
def test_both_sides_of_what_counts_as_few_tiles(edge):
    """(rows * G / 128 + B) * Hkv workgroups by what the host knows: the same tree, one request more or less."""
    for Hkv in (1, 8, 16, 24):
        B = edge // Hkv + edge % 2
        if B > 256:
            continue
        seqs = one_large(B, others=1)
        tree, chunk = plans(seqs, (Hkv, Hkv), 128)
        assert tree["tile_nsplit"] >= chunk["tile_nsplit"] > 1, (Hkv, B)


def test_large_trees_among_large_ones_are_split():
    """One long context among short ones, all with trees of the same size."""
    for heads, B, n in (((32, 8), 60, 33), ((40, 40), 20, 40), ((32, 8), 48, 40)):
        tree, chunk = plans([(65536 if b == B // 2 else 500 + 50 * b, n) for b in range(B)], heads, 128)
        assert tree["tile_nsplit"] > 4, (heads, B)


def test_drawn_batches():
    """Wherever chunks are split, trees are.  As many ranges as theirs, at least, and nowhere more than a launch holds (look)."""
    rng, split = random.Random(11), 0
    for _ in range(3000):
        Hkv = rng.choice([1, 2, 4, 8, 8, 16, 32, 40, 64])
        heads, B = (Hkv * rng.choice([1, 1, 2, 4, 8]), Hkv), rng.randint(1, 1 << rng.randint(0, 10))
        most = rng.choice([1, 2, 9, 40])
        seqs = [(rng.randint(1, 2000), rng.randint(1, most)) for _ in range(B)]
        for b in rng.sample(range(B), min(B, rng.randint(1, 3))):
            seqs[b] = (rng.randint(2000, 131072), rng.randint(33, 128))
        tree, chunk = plans(seqs, heads, rng.choice([64, 128]), rng.random() < 0.5, rng.choice([None, 131072]))
        assert tree["tile_nsplit"] >= chunk["tile_nsplit"], (heads, seqs[:5], B)
        split += chunk["tile_nsplit"] > 1
    assert split > 500


def test_workspaces_that_hold_few_ranges():
    """Two of them fit, with the 64 floats that the choice takes, or none do."""
    for heads, B in (((32, 8), 100), ((40, 40), 20), ((8, 1), 70)):
        seqs = one_large(B)
        rows = sum(n for _, n in seqs)
        few = plans(seqs, heads, 128)[0]
        used = B * heads[1] * few["few_most"] * few["nsplit"] * 129 if few["nsplit"] > 1 else 0
        for floats, ranges in ((64 + 2 * rows * heads[0] * 129, 2), (64 + 5 * rows * heads[0] * 129, 5), (64 + rows * heads[0] * 129, 1)):
            tree = plans(seqs, heads, 128, ws=4 * (used + floats))[0]
            assert tree["nsplit"] == few["nsplit"] and tree["tile_nsplit"] == ranges, (heads, B, floats)
