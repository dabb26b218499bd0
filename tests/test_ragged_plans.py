"""Host choices of the calls between a prompt and its first decode step, checked without a GPU: key ranges cover what there can be and nothing else, partial results
lie in the workspace and beside each other, launches have sizes that can be launched, whatever bounds and workspace the caller gives."""
import random

import pytest

from paper_2402_05099_amd import binding as hb

NO_BOUND = 2**31 - 1
WORKSPACES = [0, 1 << 12, 1 << 20, 64 << 20, 512 << 20, 1 << 40]
HEADS = [(1, 1), (4, 4), (8, 1), (16, 2), (32, 8), (40, 40), (64, 8), (12, 4), (9, 3), (80, 1)]


def look(rows, max_len, B, Hq, Hkv, D, max_new=None, codes=False, ws=0):
    what = f"rows {rows}, max_len {max_len}, B {B}, heads {Hq}/{Hkv}, D {D}, max_new {max_new}, workspace {ws}"
    p = hb.hg_debug_ragged_plan(rows, max_len, B, Hq, Hkv, D, max_new, codes, ws)
    assert isinstance(p, dict), f"{what}: error {p}"
    keys = max_len if max_new is not None else min(max_len, rows)      # a sequence has no more, whatever its length
    kinds = []
    if p["tiles"]:
        kinds.append((p["tile_nsplit"], p["tile_chunk"], rows * Hq, p["tile_part_O"], p["tile_part_L"]))
    else:
        assert p["tile_nsplit"] == 1
    if max_new is not None:
        kinds.append((p["nsplit"], p["chunk"], B * Hkv * p["few_most"], p["part_O"], p["part_L"]))
        assert p["few_most"] <= p["few_rows"] and p["few_most"] <= max_new * (Hq // Hkv)
        assert p["tiles"] or min(rows, max_new) * (Hq // Hkv) <= p["few_rows"], what
    else:
        assert p["tiles"] and p["nsplit"] == 1 and p["few_rows"] == 0, what
    used = []
    for n, chunk, part_rows, O, L in kinds:
        assert 1 <= n <= 256 and chunk > 0 and n * chunk >= keys, f"{what}: {n} ranges of {chunk}"
        if n == 1:
            assert O == L == -1, what
            continue
        assert chunk % 64 == 0 and (n - 1) * chunk < keys, f"{what}: {n} ranges of {chunk}, the last has no key"
        assert O % 4 == 0, f"{what}: rows are stored in pieces of 16 bytes"
        used += [(O, O + n * part_rows * D), (L, L + n * part_rows)]
    used.sort()
    assert all(a >= 0 and z <= ws // 4 for a, z in used), f"{what}: parts {used} outside the workspace"
    assert all(z <= a for (_, z), (a, _) in zip(used, used[1:])), f"{what}: parts {used} overlap"
    assert p["workgroups"] > 0 and p["workgroups"] * p["threads"] < 2**32, f"{what}: {p['workgroups']} workgroups"
    assert (p["join"] > 0) == bool(used) and p["join"] * 256 < 2**32, what
    return p


@pytest.mark.parametrize("ws", WORKSPACES)
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_under_any_bound(D, heads, ws):
    for rows in (1, 64, 130, 1024, 4096, 5000, 16384, 70000):
        for max_len in (1, 100, rows, rows + 1, 4096, 8192, 1 << 20, 1 << 30, NO_BOUND - 1, NO_BOUND):
            for B in (1, 2, 8, 9, 512):
                look(rows, max_len, B, *heads, D, ws=ws)


@pytest.mark.parametrize("D", [64, 128])
def test_a_prompt_s_bound_beyond_its_tokens_changes_nothing(D):
    for rows in (1, 130, 1024, 4096):
        want = look(rows, rows, 2, 8, 8, D, ws=512 << 20)
        for max_len in (rows + 1, 8 * rows, 1 << 30, NO_BOUND):
            assert look(rows, max_len, 2, 8, 8, D, ws=512 << 20) == want


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("ws", WORKSPACES)
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("D", [64, 128])
def test_chunks_under_any_bound(D, heads, ws, codes):
    for rows in (1, 45, 256, 3000, 20000):
        for max_new in (1, 3, 8, 64, 2048, NO_BOUND):
            for max_len in (0, 1, 515, 1280, 1281, 4096, 32768, 65536 + 33, (1 << 30) - 2):
                for B in (1, 3, 45, 512):
                    look(rows, max_len, B, *heads, D, max_new, codes, ws)


def test_drawn_calls():
    rng = random.Random(5)

    def size(most):
        return min(most, int(2 ** rng.uniform(0, most.bit_length())))

    for _ in range(20000):
        Hq, Hkv = rng.choice(HEADS)
        B, rows, ws = size(4096), size(200000), rng.choice(WORKSPACES + [size(1 << 30)])
        paged = rng.random() < 0.6
        look(rows, size((1 << 30) - 2) if paged else size(NO_BOUND), B, Hq, Hkv, rng.choice([64, 128]), size(NO_BOUND) if paged else None, rng.random() < 0.5, ws)


def test_nothing_to_do_and_refusals():
    assert hb.hg_debug_ragged_plan(0, 5, 1, 4, 4, 64)["workgroups"] == 0
    assert hb.hg_debug_ragged_plan(5, 0, 1, 4, 4, 64)["workgroups"] == 0
    assert hb.hg_debug_ragged_plan(5, 5, 0, 4, 4, 64, 1)["workgroups"] == 0
    assert hb.hg_debug_ragged_plan(5, 5, 1, 4, 3, 64) == hb.HG_ERR_UNSUPPORTED
    assert hb.hg_debug_ragged_plan(5, 5, 1, 4, 4, 32) == hb.HG_ERR_UNSUPPORTED
    assert hb.hg_debug_ragged_plan(5, -1, 1, 4, 4, 64) == hb.HG_ERR_INVALID_ARG
    assert hb.hg_debug_ragged_plan(5, (1 << 30) - 1, 1, 4, 4, 64, 1) == hb.HG_ERR_UNSUPPORTED


@pytest.mark.parametrize("ws", [0, 512 << 20, 1 << 40])
@pytest.mark.parametrize("heads", [(8, 1), (32, 8), (64, 8)])
@pytest.mark.parametrize("B", [20000, 100000, 1000000])
def test_many_sequences_of_which_few_bring_tokens(B, heads, ws):
    """A launch has fewer than 2^32 threads: the places for tiles are as many as there are sequences, whatever the tokens."""
    for rows in (1, 200, 4000):
        for max_len in (515, 4096, 65536):
            look(rows, max_len, B, *heads, 128, 200, ws=ws)
            look(rows, max_len, B, *heads, 64, 1, ws=ws)
            look(rows, max_len, B, *heads, 128, ws=ws)


def test_the_most_sequences():
    B = (1 << 20) - 1
    while not isinstance(hb.hg_debug_ragged_plan(100, 4096, B, 8, 8, 64, 200), dict):
        B -= 1
    assert B > 1000000
    look(100, 4096, B, 8, 8, 64, 200, ws=1 << 40)
    look(100, 4096, B, 8, 8, 64, 1, ws=1 << 40)
    look(100, 100, B, 8, 8, 64, ws=1 << 40)


@pytest.mark.parametrize("max_new", [None, 1])
@pytest.mark.parametrize("D", [64, 128])
def test_a_token_s_heads_lie_within_two_gibibytes(D, max_new):
    """The kernels find a head's query in its token's row by 32-bit distances."""
    most = (1 << 30) // D
    look(1, 1, 1, most, 1, D, max_new)
    assert hb.hg_debug_ragged_plan(1, 1, 1, most + 1, 1, D, max_new) == hb.HG_ERR_UNSUPPORTED


@pytest.mark.parametrize("codes", [0, 1])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_of_a_write_lie_within_32_bits(D, codes):
    """A pool without pages: the sizes are checked, and nothing would be written."""
    import ctypes
    some = ctypes.create_string_buffer(4096)      # (stands for a context and for tensors, which are not looked into)
    at = ctypes.c_void_p((ctypes.addressof(some) + 255) // 256 * 256)
    kv = hb.hg_paged_kv(at, at, at, 16, 1, 0, codes, 1.0, 1.0)
    most = (1 << 31) // D
    for Hkv, want in ((8, hb.HG_OK), (most - 1, hb.HG_OK), (most, hb.HG_ERR_UNSUPPORTED), (2 * most, hb.HG_ERR_UNSUPPORTED)):
        assert hb.lib().hg_kv_write_paged(at, at, at, Hkv * D, at, 1, ctypes.byref(kv), Hkv, D) == want


def test_the_workspace_that_calls_take_at_most():
    """the figures of include/hydragen.h"""
    rng = random.Random(1)
    for _ in range(30000):
        Hq, Hkv = rng.choice(HEADS + [(128, 1), (128, 8), (96, 96)])
        D, rows, max_len = rng.choice([64, 128]), min(400000, int(2 ** rng.uniform(0, 19))), min(131072, int(2 ** rng.uniform(0, 18)))
        B, max_new = min(2048, 2 * rows, int(2 ** rng.uniform(0, 12))), rng.choice([None, int(2 ** rng.uniform(0, 13))])
        p = look(rows, max_len, B, Hq, Hkv, D, max_new, ws=1 << 44)
        few = 4 * (D + 1) * (p["nsplit"] * B * Hkv * p["few_most"] if p["nsplit"] > 1 else 0)
        tiles = 4 * (D + 1) * (p["tile_nsplit"] * rows * Hq if p["tile_nsplit"] > 1 else 0)
        assert few <= 65 << 20 and few + tiles <= 384 << 20
