"""Key ranges of trees' tiles on the GPU, by the host (more than 256 sequences) and by the workgroups among more workgroups than the host is sure of: every test says how its call is planned, so that a
moved threshold fails it."""
import numpy as np
import pytest
import torch

import tree_plain as plain
from paper_2402_05099_amd import binding as hb
from test_gpu_ragged import DEV, context, i32, verify as check_rows
from test_gpu_trees import tree_case

pytestmark = pytest.mark.gpu
MIB = 256


def plan_of(lens, counts, heads, D, codes, max_len):
    p = hb.hg_debug_ragged_plan(sum(counts), max_len, len(lens), *heads, D, max(counts), codes, MIB << 20, tree=True)
    one = (sum(counts) * (heads[0] // heads[1]) // 128 + len(lens)) * heads[1]
    return p, one


def run(pairs, heads, D, *, max_len=None, fp32=False, **how):
    """The call against the plain form, and once more: the same bits.  Returns the plan, what the host counts as tiles, and the longest range that the workgroups have chosen."""
    Q, Qd, off, T, lens, counts, sees, masks, kv, keys, values = tree_case(pairs, *heads, D, **how)
    bound = max_len or max(lens)
    if bound > kv.page_table.shape[1] * 16:
        wide = torch.full((len(lens), -(-bound // 16)), -1, dtype=torch.int32, device=DEV)
        wide[:, :kv.page_table.shape[1]] = kv.page_table
        kv = hb.PagedKV(kv.K, kv.V, wide, 16, kv.kv_format, kv.k_scale, kv.v_scale)
    p, one = plan_of(lens, counts, heads, D, how.get("codes", False), bound)
    ctx, outs = context(MIB), []
    for _ in range(2):
        O = torch.full((T, heads[0], D), 7.0, dtype=torch.float32 if fp32 else torch.bfloat16, device=DEV)
        L = torch.full((T, heads[0]), 7.0, dtype=torch.float32, device=DEV)
        hb.hg_tree_attn_paged(ctx, Qd, i32(off.tolist()), masks, kv, i32(lens), max(counts), bound, O, L)
        torch.cuda.synchronize()
        outs.append((O, L))
    choice = int(ctx.workspace.view(torch.int32)[p["tile_part_O"] - 64]) if p["tile_nsplit"] > 1 and len(lens) <= 256 else None
    ctx.close()
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    Oref, Lref = plain.attention(Q, off, sees, keys, values, lens)
    check_rows(*outs[0], Oref, Lref, f"tree {pairs[:4]} {heads} {D} {how}", 7.0)
    return p, one, choice


@pytest.mark.parametrize("kind", ["tree", "any"])
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_ranges_by_the_host(D, codes, kind):
    """Two large trees among 298 other requests: ranges by the host's rule, sequences longer and shorter than one, one whose tree lies across a border of ranges, and one without rows."""
    pairs = [(20 + b % 60, b % 3) for b in range(296)]
    pairs[7:7], pairs[150:150], pairs[200:200], pairs[290:290] = [(4200, 40)], [(2071, 47)], [(0, 40)], [(1030, 33)]
    p, _, _ = run(pairs, (8, 2), D, codes=codes, kind=kind, fp32=kind == "any", lead=2, trail=3)
    assert len(pairs) > 256 and p["tiles"] and p["tile_nsplit"] > 1 and p["tile_chunk"] >= 1024 and p["join"] > 0
    if p["tile_chunk"] == 1088:
        assert 2071 - 47 < 2 * 1088 > 2071 - 1      # (a tree that begins in one range ends in it)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_ranges_of_a_large_tree_among_single_requests(D, codes):
    pairs = [(20 + b, b % 3) for b in range(60)]
    pairs[31] = (3000, 40)
    p, one, choice = run(pairs, (16, 16), D, codes=codes)
    assert one > 768 and p["tile_nsplit"] > 1 and p["tile_chunk"] <= choice < 3000


@pytest.mark.parametrize("kind", ["tree", "any"])
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_ranges_of_a_long_context_among_short_ones(D, codes, kind):
    """All requests have trees of 33 tokens: hundreds of tiles of few stages, eight of many."""
    pairs = [(33 + b % 50, 33) for b in range(110)]
    pairs[70] = (4000, 33)
    p, one, choice = run(pairs, (8, 8), D, codes=codes, kind=kind)
    assert one > 768 and p["tile_nsplit"] > 1 and p["tile_chunk"] <= choice < 4000


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_contexts_that_are_not_worth_a_split(D, codes):
    """A bound that is a capacity, contexts of about one length, trees of one and of several tiles, single tokens and nothing among them: one range each."""
    pairs = [(60 + b % 5, 33) for b in range(100)] + [(160, 140), (80, 1), (0, 0), (0, 33), (5, 33)]
    p, one, choice = run(pairs, (8, 8), D, codes=codes, max_len=8192, lead=1)
    assert one > 768 and p["tile_nsplit"] > 1 and choice > 8192


def test_as_many_jobs_as_there_can_be_tiles():
    """520 KV heads leave no job beside those that the tokens can make: two sequences of 33 rows and one of few."""
    p, one, choice = run([(1030, 33), (33, 33), (50, 3)], (520, 520), 64)
    assert one > 768 and p["tile_nsplit"] > 1 and choice > 1030


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_sequences_about_as_long_as_the_longest_range(D, codes):
    """A key more than the longest range makes two that are little more than half as long."""
    at = 0
    for _ in range(2):      # the range that is chosen for the first lengths, and then lengths about it (it may be chosen anew, so what is chosen is looked at again)
        near = [at + d for d in (-1, 0, 1, 2)] + [2 * at + d for d in (-1, 0, 1)] if at else [300, 700]
        p, one, choice = run([(2000, 40)] + [(x, 40) for x in near], (8, 2), D, codes=codes, kind="any")
        assert one <= 768 and p["tile_nsplit"] > 1 and p["tile_chunk"] <= choice < 2000
        at = choice


def test_a_captured_call_follows_its_lengths():
    """Replays with lengths for which the workgroups split, and with such that they don't: what eager calls give."""
    B, n, heads, D, cap = 110, 33, (8, 8), 128, 4096
    Q, Qd, off, T, lens, counts, sees, masks, kv, keys, values = tree_case([(4000 if b in (3, 70) else 90, n) for b in range(B)], *heads, D)
    o = i32(off.tolist())
    some = [[4000 if b == 70 else 90 for b in range(B)], [90] * B, [33 + b % 50 for b in range(B)], [4000 if b == 3 else b % 90 for b in range(B)], [0] * B]
    wide = torch.full((B, cap // 16), -1, dtype=torch.int32, device=DEV)
    wide[:, :kv.page_table.shape[1]] = kv.page_table
    kv = hb.PagedKV(kv.K, kv.V, wide, 16)
    p, one = plan_of(lens, counts, heads, D, False, cap)
    assert one > 768 and p["tile_nsplit"] > 1
    outs = lambda: (torch.zeros(T, heads[0], D, dtype=torch.bfloat16, device=DEV), torch.zeros(T, heads[0], device=DEV))  # noqa: E731
    ctx, other, length, got, choices = context(MIB), context(MIB), i32(some[0]), outs(), []
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    ctx.set_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        hb.hg_tree_attn_paged(ctx, Qd, o, masks, kv, length, n, cap, *got)
    for x in some + some[:2]:
        want = outs()
        hb.hg_tree_attn_paged(other, Qd, o, masks, kv, i32(x), n, cap, *want)
        length.copy_(i32(x))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        choices.append(int(ctx.workspace.view(torch.int32)[p["tile_part_O"] - 64]))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert [c < 4096 for c in choices] == [True, False, False, True, False, True, False]
    ctx.close()
    other.close()


def test_offsets_out_of_order_stay_within_the_call():
    """More tiles by the offsets than the tokens can have: some are not computed, and the call ends."""
    B, heads, D = 100, (16, 16), 64
    Q, Qd, off, T, lens, counts, sees, masks, kv, keys, values = tree_case([(1500 if b == 50 else 40, 40 if b % 10 == 0 else 1) for b in range(B)], *heads, D)
    wild = np.where(np.arange(B + 1) % 2 == 0, 0, T)
    ctx = context(MIB)
    O, L = torch.zeros(T, heads[0], D, dtype=torch.bfloat16, device=DEV), torch.zeros(T, heads[0], device=DEV)
    p, one = plan_of(lens, counts, heads, D, False, 1500)
    assert one > 768 and p["tile_nsplit"] > 1
    hb.hg_tree_attn_paged(ctx, Qd, i32(wild.tolist()), masks, kv, i32(lens), max(counts), 1500, O, L)
    torch.cuda.synchronize()
    hb.hg_tree_attn_paged(ctx, Qd, i32(off.tolist()), masks, kv, i32(lens), max(counts), 1500, O, L)
    torch.cuda.synchronize()
    Oref, Lref = plain.attention(Q, off, sees, keys, values, lens)
    check_rows(O, L, Oref, Lref, "behind a call with offsets out of order", 7.0)
    ctx.close()
