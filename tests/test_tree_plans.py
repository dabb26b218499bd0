"""Host choices of the attention of drafted trees, checked without a GPU: whatever bounds and workspace the caller gives, partial results lie in the workspace and beside each other, there are
workgroups for every tile, and launches have sizes that can be launched."""
import random

import pytest

from paper_2402_05099_amd import binding as hb

HEADS = [(1, 1), (4, 4), (8, 1), (16, 2), (32, 8), (40, 40), (64, 8), (12, 4), (9, 3), (80, 1), (600, 600)]


def look(rows, max_len, B, Hq, Hkv, D, max_new, codes, ws):
    what = f"rows {rows}, max_len {max_len}, B {B}, heads {Hq}/{Hkv}, D {D}, max_new {max_new}, workspace {ws}"
    p = hb.hg_debug_ragged_plan(rows, max_len, B, Hq, Hkv, D, max_new, codes, ws, tree=True)
    assert isinstance(p, dict), f"{what}: error {p}"
    G = Hq // Hkv
    most = min(rows, max_new) * G
    assert bool(p["tiles"]) == (most > p["few_rows"]), what
    used = []
    for n, chunk, part_rows, O, L in ((p["tile_nsplit"], p["tile_chunk"], rows * Hq, p["tile_part_O"], p["tile_part_L"]), (p["nsplit"], p["chunk"], B * Hkv * p["few_most"], p["part_O"], p["part_L"])):
        assert 1 <= n <= 256 and chunk > 0 and n * chunk >= max_len, what
        if n == 1:
            assert O == L == -1, what
            continue
        assert chunk % 64 == 0 and O % 4 == 0, what
        used += [(O, O + n * part_rows * D), (L, L + n * part_rows)]
    one = (rows * G // 128 + B) * Hkv      # workgroups with a range each
    chosen = p["tile_nsplit"] > 1 and B <= 256 and one <= 768 and max_len >= 1024      # ... or more of them, as the device chooses
    if chosen:
        assert p["tile_nsplit"] <= 64, f"{what}: the device looks at 64 ranges at most"
        used.append((p["tile_part_O"] - 64, p["tile_part_O"]))      # the choice that it leaves for the join
    used.sort()
    assert all(a >= 0 and z <= ws // 4 for a, z in used), f"{what}: parts {used} outside the workspace"
    assert all(z <= a for (_, z), (a, _) in zip(used, used[1:])), f"{what}: parts {used} overlap"
    assert p["workgroups"] > 0 and p["workgroups"] * p["threads"] < 2**32, what
    if p["tiles"]:
        assert p["workgroups"] >= one * (1 if chosen else p["tile_nsplit"]), f"{what}: a tile has no workgroup"
    assert (p["join"] > 0) == (p["nsplit"] > 1 or p["tile_nsplit"] > 1) and p["join"] * 256 < 2**32, what
    return p


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("ws", [0, 200, 1 << 12, 1 << 20, 64 << 20, 1 << 40])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("D", [64, 128])
def test_trees_under_any_bound(D, heads, ws, codes):
    for rows in (1, 45, 256, 3000, 20000):
        for max_new in (1, 8, 33, 64, 1024, 2**31 - 1):
            for max_len in (0, 1, 515, 1023, 1024, 4096, 65536 + 33, (1 << 30) - 2):
                for B in (1, 3, 64, 65, 256, 512):
                    look(rows, max_len, B, *heads, D, max_new, codes, ws)


def test_drawn_calls():
    rng = random.Random(7)
    for _ in range(4000):
        Hkv = rng.randint(1, 64)
        look(rng.randint(1, 1 << rng.randint(0, 18)), rng.randint(0, 1 << rng.randint(0, 29)), rng.randint(1, 1 << rng.randint(0, 12)), Hkv * rng.randint(1, 16), Hkv, rng.choice([64, 128]),
             rng.randint(1, 1 << rng.randint(0, 30)), rng.random() < 0.5, rng.choice([0, 1 << rng.randint(0, 34)]))


def test_what_the_cases_run_as():
    """48 requests, 32/8 heads: tiles of one range each, the longest first, and few rows in ranges; three behind long documents: ranges chosen on the device."""
    p = look(2328, 4192, 48, 32, 8, 128, 96, False, 512 << 20)
    assert p["tiles"] and p["tile_nsplit"] == 1 and p["nsplit"] > 1
    p = look(192, 65600, 3, 64, 8, 128, 64, False, 512 << 20)
    assert p["tiles"] and p["tile_nsplit"] > 8
    p = look(4, 64, 4, 4, 4, 64, 1, False, 512 << 20)
    assert not p["tiles"] and p["join"] == 0
