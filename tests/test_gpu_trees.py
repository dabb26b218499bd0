"""A decode step over trees of drafted tokens on the GPU: masks, attention over the paged cache, verification, the accepted rows' move, against the plain forms of
tree_plain.py in 64 bits.  Attention is held to the gates of parity.py (weights and results are rounded to bf16 as in the decode kernels); the rest is whole numbers and copies, equal bit for bit."""
import math

import numpy as np
import pytest
import torch

import tree_plain as plain
from paper_2402_05099_amd import binding as hb
from test_gpu_ragged import DEV, HEADS, NAN, context, i32, make_cache, offsets, rand, verify as check_rows

pytestmark = pytest.mark.gpu


def random_parents(r, n, width, wild=0.0):
    """each token's parent among the `width` before it; some are no parent at all"""
    up = [-1] + [int(t - 1 - r.integers(0, min(t, width))) for t in range(1, n)]
    return [int(r.choice([-1, -5, t, t + 3, 1 << 30])) if r.random() < wild else p for t, p in enumerate(up)][:n]


# ---- masks -------------------------------------------------------------------------------------------------------------------

def run_masks(counts, width, *, lead=0, trail=0, extra=0, wild=0.0, max_new=None, depth=True, seed=0):
    r = np.random.default_rng(seed)
    ups = [random_parents(r, n, width, wild) for n in counts]
    off = offsets(counts, lead)
    T, most = int(off[-1]) + trail, max(list(counts) + [0]) if max_new is None else max_new
    count = -(-min(most, T) // 32) + extra
    parents = np.full(T, 12345, dtype=np.int64)
    masks, want, deep = [np.full((T, count), 77, dtype=np.int32) for _ in range(2)], None, np.full(T, 77)
    want = masks[1]
    for b, up in enumerate(ups):
        a, z, take = int(off[b]), int(off[b + 1]), min(len(up), most)
        parents[a:z] = up
        m = plain.follows(up)[:take, :take]
        want[a:a + take] = plain.words(m, count)
        deep[a:a + take] = m.sum(1) - 1
    got, d = torch.tensor(masks[0], device=DEV), torch.full((T,), 77, dtype=torch.int32, device=DEV) if depth else None
    ctx = context()
    hb.hg_tree_masks(ctx, i32(parents.tolist()), i32(off.tolist()), most, got, d)
    torch.cuda.synchronize()
    assert np.array_equal(got.cpu().numpy(), want)
    if depth:
        assert d.tolist() == deep.tolist()
    ctx.close()


@pytest.mark.parametrize("width", [1, 2, 7, 1 << 20])
def test_masks_of_small_trees(width):
    run_masks([0, 1, 2, 3, 31, 32, 33, 63, 64, 5, 0], width, lead=3, trail=2)
    run_masks([64] * 9, width, extra=2)
    run_masks([4, 1, 30], width, depth=False)


@pytest.mark.parametrize("width", [1, 3, 40, 1 << 20])
def test_masks_of_large_trees(width):
    run_masks([65, 0, 64, 127, 128, 129, 1, 200], width, lead=2, trail=5)
    run_masks([1024, 1000, 961, 3], width, extra=1)


def test_masks_of_tokens_without_a_parent():
    run_masks([40, 64, 3], 5, wild=0.4)
    run_masks([700, 64, 100], 9, wild=0.2)


@pytest.mark.parametrize("most", [1, 20, 64, 65, 130])
def test_masks_of_tokens_behind_the_bound_are_left(most):
    run_masks([200, 20, 64, 65, 0], 4, max_new=most)


def test_masks_of_many_sequences():
    run_masks([i % 9 for i in range(700)], 3)


# ---- attention ---------------------------------------------------------------------------------------------------------------

def tree_case(pairs, Hq, Hkv, D, *, ps=16, codes=False, lead=0, trail=0, fused=False, gain=1.0, seed=0, kind="tree", extra=0, far=0):
    """pairs: (rows in the cache with the new ones, new tokens).  kind: "tree" (ancestors), "chain", or "any" (random bits, rows without one among them)."""
    g = torch.Generator().manual_seed(seed)
    r = np.random.default_rng(seed + 1)
    lens, counts = [x for x, _ in pairs], [n for _, n in pairs]
    off = offsets(counts, lead)
    T = int(off[-1]) + trail
    scales = (0.02, 0.015)
    Kp, Vp, table, keys, values = make_cache(g, lens, Hkv, D, ps, codes, scales, far=far)
    x = rand(g, T, Hq + (3 if fused else 0), D, gain=gain)
    sees, count = [], max(1, -(-max(counts + [0]) // 32)) + extra
    bits = np.full((T, count), -1, dtype=np.int32)
    for b, n in enumerate(counts):
        if kind == "any":
            m = r.random((n, n)) < 0.3
            m[r.random(n) < 0.2] = False
        else:
            m = plain.follows(random_parents(r, n, 1 if kind == "chain" else 4))
        sees.append(m)
        wide = np.ones((n, 32 * count), dtype=bool)      # (bits behind the tokens count for nothing)
        wide[:, :n] = m
        bits[int(off[b]):int(off[b + 1])] = plain.words(wide, count)
    kv = hb.PagedKV(K=Kp, V=Vp, page_table=table, page_size=ps, kv_format=hb.HG_KV_E4M3 if codes else hb.HG_KV_BF16, k_scale=scales[0], v_scale=scales[1])
    return x[:, :Hq], x.to(DEV)[:, :Hq], off, T, lens, counts, sees, torch.tensor(bits, device=DEV), kv, keys, values


def run_attn(pairs, heads, D, *, fp32=False, lse=True, scale=0.0, max_new=None, max_len=None, mib=0, ctx=None, **how):
    Q, Qd, off, T, lens, counts, sees, masks, kv, keys, values = tree_case(pairs, *heads, D, **how)
    O = torch.full((T, heads[0], D), 7.0, dtype=torch.float32 if fp32 else torch.bfloat16, device=DEV)
    L = torch.full((T, heads[0]), 7.0, dtype=torch.float32, device=DEV) if lse else None
    own = ctx or context(mib)
    hb.hg_tree_attn_paged(own, Qd, i32(off.tolist()), masks, kv, i32(lens), max(counts + [0]) if max_new is None else max_new,
                          max(lens + [0]) if max_len is None else max_len, O, L, scale)
    torch.cuda.synchronize()
    seen = lens if max_len is None else [min(x, max_len) for x in lens]
    Oref, Lref = plain.attention(Q, off, sees, keys, values, seen, scale or None, max_new)
    check_rows(O, L, Oref, Lref, f"tree {pairs[:6]} {heads} {D} {how}", 7.0)
    if ctx is None:
        own.close()


MIXED = [(1, 1), (40, 0), (17, 17), (300, 33), (0, 0), (65, 1), (3, 5), (0, 4), (129, 64), (64, 64), (200, 2), (95, 31), (97, 32)]      # (3, 5), (0, 4): tokens without rows


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", HEADS)
def test_trees_of_every_kind(heads, D, codes):
    run_attn(MIXED, heads, D, codes=codes, lead=2, trail=3, fused=heads[0] == 10)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [(4, 4), (16, 2), (64, 8)])
def test_masks_of_any_kind(heads, D, codes):
    run_attn(MIXED, heads, D, codes=codes, kind="any", extra=2, fp32=True)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ps", [16, 64, 1024])
def test_pages_of_other_sizes(ps, D, codes):
    run_attn(MIXED, (16, 2), D, ps=ps, codes=codes, mib=64, kind="any")


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("where", list(range(-3, 36, 3)))
def test_a_tree_that_begins_anywhere_in_a_stage(where, D, codes):
    run_attn([(96 + where + 40, 40), (max(where, 0) + 7, 7), (64 + where + 100, 100)], (8, 2), D, codes=codes, kind="any")


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mib", [0, 1, 256])
def test_long_contexts_whatever_the_workspace(D, codes, mib):
    run_attn([(4100, 1), (70, 3), (3001, 40)], (16, 2), D, ps=64, codes=codes, mib=mib, fp32=True)
    run_attn([(5000, 9), (2000, 3)], (4, 4), D, ps=64, codes=codes, mib=mib, kind="any")


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_trees_of_hundreds_of_tokens(D, codes):
    run_attn([(700, 300), (257, 257), (40, 3)], (8, 2), D, codes=codes)
    run_attn([(400, 130), (257, 257)], (4, 4), D, codes=codes, kind="any", mib=64)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_tokens_and_rows_behind_the_bounds(D, codes):
    run_attn([(300, 40), (20, 7), (90, 64)], (8, 2), D, codes=codes, max_new=17)
    run_attn([(300, 40), (20, 7), (90, 64)], (8, 2), D, codes=codes, max_len=100)


# (It is up to 256 sequences, not 64, that the workgroups choose for.)
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 130, 256, 257])
def test_key_ranges_of_many_sequences(B, D, codes):
    """Up to 64 sequences the workgroups choose the ranges from the lengths; long ones among short and empty ones, trees that are tiles among those that are few rows."""
    pairs = [(max(n, (1500 if b % 7 == 0 else 40) + 13 * b % 300), n) for b in range(B) for n in [(40, 3, 0, 17, 64, 9, 33)[b % 7]]]
    run_attn(pairs, (8, 2), D, codes=codes, mib=64)
    if B < 64:
        run_attn(pairs, (8, 2), D, codes=codes, mib=1, kind="any")


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_tiles_of_sequences_without_enough_rows(D, codes):
    """Trees of more tokens than the cache has rows (a step that ran out of pages): the rows that are there are the last tokens', some or all tokens see nothing."""
    for kind in ("tree", "any"):
        run_attn([(0, 64), (5, 64), (64, 64), (33, 100), (70, 64)], (8, 2), D, codes=codes, kind=kind)
    run_attn([(0, 64), (5, 64), (1500, 64), (33, 100)], (8, 2), D, codes=codes, mib=64)
    run_attn([(40, 9), (70, 64), (0, 3)], (8, 2), D, codes=codes, max_len=0)


# (66 and 72 sequences: here too the workgroups choose.  Ranges by the host, for more than 256, are in test_gpu_tree_ranges.py.)
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_key_ranges_of_more_sequences_than_are_ordered(D, codes):
    """Two large trees behind long contexts among 64 and more others: the ranges are the host's."""
    run_attn([(3000, 40), (2500, 33)] + [(20 + b, b % 3) for b in range(64)], (8, 2), D, codes=codes, mib=64)
    run_attn([(20 + b, b % 3) for b in range(70)] + [(3000, 40), (0, 40)], (8, 2), D, codes=codes, mib=64, kind="any")


def test_many_heads_to_a_kv_head():
    run_attn([(50, 7), (300, 3), (33, 33), (9, 1)], (80, 1), 128, mib=64)
    run_attn([(50, 7), (300, 3), (33, 33), (9, 1)], (66, 2), 64, codes=True)


def test_bounds_that_are_a_capacity():
    """max_new and max_len far above what there is, as a captured step has them."""
    pairs = [(2000, 40), (0, 0), (300, 33), (1100, 64), (5, 1)]
    Q, Qd, off, T, lens, counts, sees, masks, kv, keys, values = tree_case(pairs, 16, 2, 128)
    wide = torch.full((len(pairs), 8192), -1, dtype=torch.int32, device=DEV)
    wide[:, :kv.page_table.shape[1]] = kv.page_table
    kv = hb.PagedKV(K=kv.K, V=kv.V, page_table=wide, page_size=16)
    Oref, Lref = plain.attention(Q, off, sees, keys, values, lens)
    for mib in (0, 16, 256):
        ctx = context(mib)
        O, L = torch.full((T, 16, 128), 7.0, device=DEV), torch.full((T, 16), 7.0, device=DEV)
        bits = torch.cat([masks, torch.zeros(T, 32 - masks.shape[1], dtype=torch.int32, device=DEV)], 1).contiguous()
        hb.hg_tree_attn_paged(ctx, Qd, i32(off.tolist()), bits, kv, i32(lens), 1024, 131072, O, L)
        torch.cuda.synchronize()
        check_rows(O, L, Oref, Lref, f"bounds of a capacity, {mib} MiB", 7.0)
        ctx.close()


@pytest.mark.parametrize("D", [64, 128])
def test_results_in_fp32_without_lse_peaked(D):
    run_attn(MIXED, (8, 2), D, lse=False, scale=0.3)
    run_attn(MIXED, (8, 2), D, fp32=True, gain=6.0)
    run_attn([(300, 200)], (8, 2), D, fp32=True, gain=6.0)


def test_a_pool_that_passes_two_gigabytes():
    run_attn([(300, 33), (65, 1)], (16, 2), 128, ps=1024, far=4200)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [(4, 4), (16, 2)])
def test_chains_are_chunks(heads, D, codes):
    """The same rows seen.  Weights are rounded to bf16 on either side, by 2^-8 of themselves at most, and sum to one with values of at most max |v|; sums of up to 1000 weights in fp32
    are off by 1000 * 2^-24 = 6e-5 of themselves at most, and so are their logarithms."""
    Q, Qd, off, T, lens, counts, sees, masks, kv, keys, values = tree_case([(300, 33), (65, 1), (17, 17), (1000, 200), (90, 0)], *heads, D, codes=codes, kind="chain")
    outs = []
    ctx = context(64)
    for f, more in ((hb.hg_tree_attn_paged, (masks,)), (hb.hg_chunk_attn_paged, ())):
        O, L = torch.zeros(T, heads[0], D, dtype=torch.float32, device=DEV), torch.zeros(T, heads[0], device=DEV)
        f(ctx, Qd, i32(off.tolist()), *more, kv, i32(lens), max(counts), max(lens), O, L)
        outs.append((O, L))
    torch.cuda.synchronize()
    most = max(float(v.abs().max()) for v in values)
    assert (outs[0][1] - outs[1][1]).abs().max() <= 2 * 6e-5 and (outs[0][0] - outs[1][0]).abs().max() <= 2 * 2 ** -8 * most
    ctx.close()


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,context_rows", [(9, 150), (90, 150), (9, 1500), (90, 1500)])      # (behind 1500 rows in several ranges of keys)
@pytest.mark.parametrize("what", ["k", "v", "inf"])
def test_values_that_are_not_finite_reach_only_those_that_see_them(what, n, context_rows, D, codes):
    if what == "inf" and codes:
        return      # (the codes have no infinities)
    heads, lens = (8, 2), [n + context_rows, n + 3]
    Q, Qd, off, T, lens, counts, sees, masks, kv, keys, values = tree_case([(x, n) for x in lens], *heads, D, codes=codes)
    bad = n // 2      # a token of the tree whose row is spoiled: it and those that follow from it have NaN or infinity
    for b in range(2):
        j = lens[b] - n + bad
        row = int(kv.page_table[b, j // 16]) * 16 + j % 16
        if codes:
            (kv.K if what == "k" else kv.V)[row] = 0x7F
        else:
            (kv.K if what == "k" else kv.V)[row] = math.inf if what == "inf" else NAN
    outs = []
    for mib in (0, 64):
        ctx = context(mib)
        O, L = torch.zeros(T, 8, D, dtype=torch.float32, device=DEV), torch.zeros(T, 8, device=DEV)
        hb.hg_tree_attn_paged(ctx, Qd, i32(off.tolist()), masks, kv, i32(lens), n, max(lens), O, L)
        torch.cuda.synchronize()
        outs.append((O.cpu(), L.cpu()))
        ctx.close()
    Oref, Lref = plain.attention(Q, off, sees, keys, values, lens)
    for O, L in outs:
        for b in range(2):
            hit = torch.tensor(sees[b][:, bad])
            o, l = O[int(off[b]):int(off[b + 1])], L[int(off[b]):int(off[b + 1])]
            assert torch.isfinite(o[~hit]).all() and torch.isfinite(l[~hit]).all()
            assert not torch.isfinite(o[hit]).any()
            keep = torch.zeros(T, dtype=torch.bool)
            keep[int(off[b]):int(off[b + 1])] = ~hit
            check_rows(O[keep], L[keep], Oref[keep], Lref[keep], "beside a spoiled row")


def test_tree_attention_in_a_graph_and_on_a_stream():
    Q, Qd, off, T, lens, counts, sees, masks, kv, keys, values = tree_case([(900, 33), (65, 1), (300, 90)], 16, 2, 128)
    ctx = context(64)
    o, ln = i32(off.tolist()), i32(lens)
    want, got = [(torch.zeros(T, 16, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(T, 16, device=DEV)) for _ in range(2)]
    hb.hg_tree_attn_paged(ctx, Qd, o, masks, kv, ln, 90, 900, *want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    ctx.set_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        hb.hg_tree_attn_paged(ctx, Qd, o, masks, kv, ln, 90, 900, *got)
    for _ in range(3):
        got[0].zero_()
        got[1].zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    ctx.close()


@pytest.mark.parametrize("V", [3000, 98500])
def test_a_whole_step_in_a_graph(V):
    """Masks, attention, verification and the move captured on a stream of their own, replayed with eager work and other lengths between: the results of eager calls."""
    g, r = torch.Generator().manual_seed(5), np.random.default_rng(5)
    Hq, Hkv, D, ps, B, n = 8, 2, 128, 16, 6, 70
    T = B * n
    Kp, Vp, table, _, _ = make_cache(g, [1300] * B, Hkv, D, ps, False)
    first = [(Kp.clone(), Vp.clone()) for _ in range(2)]
    Q = rand(g, T, Hq, D).to(DEV)
    parents, off = i32(sum([random_parents(r, n, 4) for _ in range(B)], [])), i32(list(range(0, T + 1, n)))
    z = torch.randn(T, V, generator=g) * 4
    target, draft = torch.softmax(z, 1).to(DEV), torch.softmax(z + torch.randn(T, V, generator=g), 1).to(DEV)
    tokens, u, un = torch.multinomial(draft, 1)[:, 0].to(torch.int32), torch.rand(T, generator=g).to(DEV), torch.rand(B, generator=g).to(DEV)
    lens = [i32([n + int(x) for x in r.integers(0, 1230, B)]) for _ in range(4)]
    ctx = context(64)

    def step(kv, length, out):
        hb.hg_tree_masks(ctx, parents, off, n, out[0], out[1])
        hb.hg_tree_attn_paged(ctx, Q, off, out[0], kv[0], length, n, 1300, out[2], out[3])
        hb.hg_tree_verify(ctx, tokens, parents, off, n, target, draft, u, un, out[4], out[5], out[6])
        hb.hg_tree_keep_paged(ctx, kv, off, out[4], out[5], length, n, out[7])

    def buffers():
        e = lambda *shape, dtype=torch.int32: torch.zeros(*shape, dtype=dtype, device=DEV)  # noqa: E731
        return [e(T, 3), e(T), e(T, Hq, D, dtype=torch.bfloat16), e(T, Hq, dtype=torch.float32), e(T), e(B), e(B), e(B)]

    pools = [(k.clone(), v.clone()) for k, v in first]
    kv = [hb.PagedKV(k, v, table, ps) for k, v in pools]
    out, length = buffers(), lens[0].clone()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    ctx.set_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(kv, length, out)
    ctx.set_stream(None)
    for x in lens:
        again = [(k.clone(), v.clone()) for k, v in first]
        want = buffers()
        step([hb.PagedKV(k, v, table, ps) for k, v in again], x, want)
        for (k, v), (k0, v0) in zip(pools, first):
            k.copy_(k0)
            v.copy_(v0)
        length.copy_(x)
        for o in out:
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
        for a, b in zip(sum(pools, ()), sum(again, ())):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    ctx.close()


# ---- verification ------------------------------------------------------------------------------------------------------------

def run_verify(counts, V, *, dtype=torch.float32, drafts=True, width=3, sharp=0.5, lead=0, trail=0, pad=0, max_new=None, seed=0, spoil=None, near=0.7, peaked=False):
    """near: how much of the drafts' probabilities is the target's"""
    r = np.random.default_rng(seed)
    off = offsets(counts, lead)
    T, B, most = int(off[-1]) + trail, len(counts), max(list(counts) + [0]) if max_new is None else max_new
    draw = (lambda: np.exp(6 * r.standard_normal((T, V)))) if peaked else (lambda: r.dirichlet(np.full(V, sharp), T) if V <= 64 else r.random((T, V)) ** 8)
    P = draw()
    P /= P.sum(1, keepdims=True)
    other = draw()
    Q = near * P + (1 - near) * other / other.sum(1, keepdims=True)
    P, Q = (torch.tensor(x).to(dtype) for x in (P, Q))
    parents, tokens = np.full(T, -1), np.zeros(T, dtype=np.int64)
    for b, n in enumerate(counts):
        a = int(off[b])
        up = random_parents(r, n, width, 0.03)
        parents[a:a + n] = up
        for t in range(1, n):
            p = plain.parents_of(t, up)
            w = Q[a + (p or 0)].double().numpy()
            tokens[a + t] = r.choice(V, p=w / w.sum()) if r.random() < 0.95 else r.integers(-3, V + 3)
    u, un = torch.tensor(r.random(T), dtype=torch.float32).clamp(max=1 - 2 ** -24), torch.tensor(r.random(B), dtype=torch.float32).clamp(max=1 - 2 ** -24)
    if spoil:
        spoil(P, Q, u, un, off)

    def on_device(x):      # rows `pad` elements further apart than they are long, from an odd place on
        if not pad:
            return x.to(DEV)
        wide = torch.full((T, V + pad), NAN, dtype=dtype, device=DEV)
        wide[:, pad // 2:pad // 2 + V] = x.to(DEV)
        return wide[:, pad // 2:pad // 2 + V]

    Pd, Qd, got = on_device(P), on_device(Q) if drafts else None, []
    for mib in (0, 1) if V >= 98304 else (0,):      # (with a workspace the first sum over a large vocabulary is shared out)
        path, kept, nxt = (torch.full((k,), 77, dtype=torch.int32, device=DEV) for k in (T, B, B))
        ctx = context(mib)
        hb.hg_tree_verify(ctx, i32(tokens.tolist()), i32(parents.tolist()), i32(off.tolist()), most, Pd, Qd, u.to(DEV), un.to(DEV), path, kept, nxt)
        torch.cuda.synchronize()
        got.append((path, kept, nxt))
        ctx.close()
    want_path, want_kept, want_next = np.full(T, 77), [], []
    for b, n in enumerate(counts):
        a, take = int(off[b]), min(n, most)
        at = slice(a, a + take)
        p, y = plain.verify(tokens[at], parents[at], P[at].double().numpy(), Q[at].double().numpy() if drafts else None, u[at].numpy(), un[b])
        want_path[at] = p + [-1] * (take - len(p))
        want_kept.append(len(p))
        want_next.append(y)
    for path, kept, nxt in got:
        assert kept.tolist() == want_kept
        assert path.tolist() == want_path.tolist()
        assert nxt.tolist() == want_next
    return want_kept


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("drafts", [True, False])
@pytest.mark.parametrize("V", [1, 2, 5, 7, 8, 9, 63, 64, 65, 511, 512, 513, 1000])
def test_verification_over_small_vocabularies(V, drafts, dtype):
    kept = run_verify([0, 1, 2, 3, 9, 31, 33, 64, 5, 12] * 3, V, drafts=drafts, dtype=dtype, lead=2, trail=3, seed=V)
    if V <= 64:
        assert max(kept) > 1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("drafts", [True, False])
@pytest.mark.parametrize("V", [4095, 4096, 8192, 8193, 16387, 32000, 131072 + 5])
def test_verification_over_large_vocabularies(V, drafts, dtype):
    run_verify([1, 7, 0, 12] if V > 100000 else [1, 7, 0, 30, 12], V, drafts=drafts, dtype=dtype, seed=V, width=5, near=0.3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("drafts", [True, False])
@pytest.mark.parametrize("V", [300, 8190, 8200, 98305])
def test_verification_where_few_tokens_have_nearly_all(V, drafts, dtype):
    kept = run_verify([1, 7, 0, 30, 12, 64, 33, 20], V, drafts=drafts, dtype=dtype, seed=V, width=3, near=0.9, peaked=True)
    assert max(kept) > 1


@pytest.mark.parametrize("drafts", [True, False])
def test_verification_over_more_groups_than_the_filter_tells_apart(drafts):
    run_verify([6, 1, 9], 300001, drafts=drafts, near=0.9, peaked=True)


@pytest.mark.parametrize("drafts", [True, False])
@pytest.mark.parametrize("width", [1, 2, 1 << 20])
def test_verification_of_large_trees(width, drafts):
    run_verify([1024, 65, 128, 700], 40, drafts=drafts, width=width, near=0.98)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad", [1, 3, 8, 21])
def test_rows_that_lie_further_apart(pad, dtype):
    run_verify([5, 9, 1, 33], 77, dtype=dtype, pad=pad, drafts=True)
    run_verify([5, 9, 1, 33], 1030, dtype=dtype, pad=pad, drafts=False)


def test_tokens_behind_the_bound_are_not_looked_at():
    run_verify([40, 3, 0, 17, 16], 30, max_new=16, near=0.95, width=1)


def test_verification_of_many_sequences():
    run_verify([i % 6 for i in range(900)], 12, near=0.8)


@pytest.mark.parametrize("drafts", [True, False])
def test_probabilities_that_are_no_numbers(drafts):
    def spoil(P, Q, u, un, off):
        P[::2, 3] = NAN
        P[1::3, 5] = math.inf
        P[::3, 7] = -1.0
        Q[::2, 4] = NAN
        Q[1::3, 6] = math.inf
    run_verify([9, 17, 3, 30], 20, drafts=drafts, spoil=spoil)


@pytest.mark.parametrize("drafts", [True, False])
def test_rows_that_have_nothing(drafts):
    def nothing(P, Q, u, un, off):
        P[:] = 0

    def same(P, Q, u, un, off):      # what is left after a refusal is nothing: the draw is from p
        P[:] = 0.0
        P[:, 2] = 0.5
        Q[:] = P
        Q[:, 2] = 1.0
    for V in (2000, 98311):
        run_verify([9, 17, 1], V, drafts=drafts, spoil=nothing)
        run_verify([9, 17, 1], V, drafts=drafts, spoil=same)


@pytest.mark.parametrize("at", [0.0, 2 ** -24, 0.5, 1 - 2 ** -24])
@pytest.mark.parametrize("V", [3, 600, 9000, 100000])
def test_random_numbers_at_the_ends(at, V):
    def spoil(P, Q, u, un, off):
        u[:], un[:] = at, at
        P[:, :2] = 0
        P[:, -1] = 0
        P[:, V // 2] = 0.3
    for drafts in (True, False):
        run_verify([9, 17, 1, 40], V, drafts=drafts, spoil=spoil)


@pytest.mark.parametrize("drafts", [True, False])
def test_what_comes_out_is_distributed_as_the_target_says(drafts):
    """The token behind the first, over 40000 sequences of one distribution and three siblings: each of the seven counts is binomial, and within 5 standard deviations of its mean but for a
    chance of 7 * 6e-7."""
    B, V, n = 40000, 7, 4
    r = np.random.default_rng(11)
    p, q = r.dirichlet(np.ones(V)), r.dirichlet(np.ones(V))
    tokens = np.zeros((B, n), dtype=np.int64)
    for b in range(B):
        tokens[b, 1:] = r.choice(V, 3, p=q) if drafts else r.choice(V, 3, replace=False, p=q)
    P = torch.tensor(p, dtype=torch.float32, device=DEV).expand(B * n, V).contiguous()
    Q = torch.tensor(q, dtype=torch.float32, device=DEV).expand(B * n, V).contiguous() if drafts else None
    g = torch.Generator(device=DEV).manual_seed(3)
    u, un = torch.rand(B * n, generator=g, device=DEV), torch.rand(B, generator=g, device=DEV)
    path, kept, nxt = (torch.zeros(x, dtype=torch.int32, device=DEV) for x in (B * n, B, B))
    ctx = context()
    hb.hg_tree_verify(ctx, torch.tensor(tokens.reshape(-1), dtype=torch.int32, device=DEV), i32([-1, 0, 0, 0] * B), i32(list(range(0, B * n + 1, n))), n, P, Q, u, un, path, kept, nxt)
    torch.cuda.synchronize()
    second = path.view(B, n)[:, 1].cpu().numpy()
    first = np.where(second >= 0, tokens[np.arange(B), np.maximum(second, 0)], nxt.cpu().numpy())
    counts = np.bincount(first, minlength=V)
    assert np.all(np.abs(counts - B * p) <= 5 * np.sqrt(B * p * (1 - p)) + 1), (counts, B * p)
    assert 0.3 < (second >= 0).mean() < 1
    ctx.close()


@pytest.mark.parametrize("width", [1, 3, 50])
def test_greedy_verification(width):
    r = np.random.default_rng(width)
    counts = [0, 1, 2, 30, 64, 65, 300, 1024, 7]
    off = offsets(counts, 1)
    T, B = int(off[-1]) + 2, len(counts)
    tokens, says = r.integers(0, 3, T), r.integers(0, 3, T)
    parents = np.full(T, -1)
    for b, n in enumerate(counts):
        parents[int(off[b]):int(off[b + 1])] = random_parents(r, n, width, 0.02)
    path, kept, nxt = (torch.full((x,), 77, dtype=torch.int32, device=DEV) for x in (T, B, B))
    ctx = context()
    hb.hg_tree_verify(ctx, i32(tokens.tolist()), i32(parents.tolist()), i32(off.tolist()), 1000, i32(says.tolist()), None, None, None, path, kept, nxt)
    torch.cuda.synchronize()
    want = np.full(T, 77)
    for b, n in enumerate(counts):
        at = slice(int(off[b]), int(off[b]) + min(n, 1000))
        p, y = plain.verify(tokens[at], parents[at], says[at], None, None, None)
        want[at] = p + [-1] * (min(n, 1000) - len(p))
        assert (kept[b].item(), nxt[b].item()) == (len(p), y)
    assert path.tolist() == want.tolist()
    ctx.close()


# ---- the accepted rows' move -------------------------------------------------------------------------------------------------

def run_keep(pairs, *, Hkv=2, D=128, ps=16, codes=False, layers=1, max_new=None, wild=0.0, holes=False, seed=0, lead=0, most_kept=None):
    r = np.random.default_rng(seed)
    lens, counts = [x for x, _ in pairs], [n for _, n in pairs]
    off = offsets(counts, lead)
    T, B, most = int(off[-1]) + 2, len(pairs), max(counts + [0]) if max_new is None else max_new
    need = [-(-max(x, 0) // ps) for x in lens]
    n_pages, stride = sum(need) + 2, max(need + [1])
    table, order, at = np.full((B, stride), -9), r.permutation(n_pages), 0
    for b in range(B):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    if holes:
        table[r.random(table.shape) < 0.2] = -1
        table[r.random(table.shape) < 0.2] = n_pages
    path, kept = np.full(T, 99), []
    for b, n in enumerate(counts):
        a = int(r.integers(0, n + 1)) if most_kept is None else min(n, most_kept)
        p = np.sort(r.permutation(n)[:a])
        p = np.where(r.random(a) < wild, r.choice([-1, n, n + 5, 1 << 30], a), p) if n else p
        path[int(off[b]):int(off[b]) + a] = p
        kept.append(a if r.random() < 0.9 or wild == 0 else a + 5)
    dt = torch.uint8 if codes else torch.bfloat16
    pools = [torch.tensor(r.integers(0, 256, (n_pages * ps, Hkv, D * (1 if codes else 2))), dtype=torch.uint8) for _ in range(2 * layers)]
    dev = [p.to(DEV).view(dt) for p in pools]
    t = torch.tensor(table, dtype=torch.int32, device=DEV)
    kvs = [hb.PagedKV(dev[2 * i], dev[2 * i + 1], t, ps, hb.HG_KV_E4M3 if codes else hb.HG_KV_BF16, 0.1, 0.1) for i in range(layers)]
    grown = torch.full((B,), 77, dtype=torch.int32, device=DEV)
    ctx = context()
    hb.hg_tree_keep_paged(ctx, kvs, i32(off.tolist()), i32(path.tolist()), i32(kept), i32(lens), most, grown)
    torch.cuda.synchronize()
    want, lengths = plain.keep([p.numpy() for p in pools], table, ps, off, path, kept, lens, most)
    for got, w in zip(dev, want):
        assert np.array_equal(got.view(torch.uint8).cpu().numpy(), w)
    assert grown.tolist() == lengths
    ctx.close()


KEEP = [(1, 1), (40, 0), (17, 17), (300, 33), (0, 0), (65, 1), (3, 5), (0, 4), (129, 64), (64, 64), (512, 2), (33, 20)]


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hkv", [1, 2, 8, 40])
def test_accepted_rows_move_together(Hkv, D, codes):
    run_keep(KEEP, Hkv=Hkv, D=D, codes=codes, lead=1)


@pytest.mark.parametrize("ps", [16, 64, 1024])
@pytest.mark.parametrize("layers", [1, 3, 128])
def test_accepted_rows_of_many_layers(layers, ps):
    run_keep(KEEP if layers < 100 else KEEP[:4], layers=layers, ps=ps, seed=layers)


def test_more_rows_than_are_looked_up_at_once():
    run_keep([(1024, 1024), (700, 600), (300, 257)])
    run_keep([(1024, 1024), (700, 600)], most_kept=513)


def test_paths_and_tables_with_holes():
    run_keep(KEEP, wild=0.3)
    run_keep(KEEP, holes=True)
    run_keep(KEEP, max_new=16)


# ---- calls with nothing in them, offsets that leave the tensors ----------------------------------------------------------------

def test_calls_without_tokens_and_without_sequences():
    ctx = context(1)
    e = lambda *shape, dtype=torch.int32: torch.full(shape, 7, dtype=dtype, device=DEV)  # noqa: E731
    bf, f32 = torch.bfloat16, torch.float32
    for B in (0, 3):
        off, len_, table, kept, nxt, grown = i32([0] * (B + 1)), i32([5] * B), torch.zeros(B, 4, dtype=torch.int32, device=DEV), e(B), e(B), e(B)
        kv = hb.PagedKV(e(64, 2, 64, dtype=bf), e(64, 2, 64, dtype=bf), table, 16)
        hb.hg_tree_masks(ctx, e(0), off, 8, e(0, 1), e(0))
        hb.hg_tree_attn_paged(ctx, e(0, 4, 64, dtype=bf), off, e(0, 1), kv, len_, 8, 16, e(0, 4, 64, dtype=bf), e(0, 4, dtype=f32))
        hb.hg_tree_verify(ctx, e(0), e(0), off, 8, e(0, 100, dtype=f32), e(0, 100, dtype=f32), e(0, dtype=f32), e(B, dtype=f32), e(0), kept, nxt)
        assert kept.tolist() == [0] * B and nxt.tolist() == [-1] * B
        hb.hg_tree_keep_paged(ctx, [kv], off, e(0), kept, len_, 8, grown)
        assert grown.tolist() == [5] * B and torch.all(kv.K == 7)
    ctx.close()


def test_offsets_behind_the_tensors_end_with_them():
    """q_off says more tokens than there are rows: those that are there are a smaller tree's."""
    r, g, T, V = np.random.default_rng(3), torch.Generator().manual_seed(3), 30, 50
    off, clamped = [0, 12, 45, 90], [0, 12, 30, 30]
    ups = [random_parents(r, n, 3) for n in (12, 18)]
    parents, tokens, says = i32(sum(ups, [])), i32(r.integers(0, 2, T).tolist()), i32(r.integers(0, 2, T).tolist())
    lens = [40, 60, 33]
    Kp, Vp, table, keys, values = make_cache(g, lens, 2, 64, 16, False)
    kv, Q = hb.PagedKV(Kp, Vp, table, 16), rand(g, T, 4, 64)
    got = []
    for o in (off, clamped):
        ctx = context()
        m, d, O, L = torch.zeros(T, 2, dtype=torch.int32, device=DEV), i32([0] * T), torch.zeros(T, 4, 64, device=DEV), torch.zeros(T, 4, device=DEV)
        path, kept, nxt, grown = i32([7] * T), i32([7] * 3), i32([7] * 3), i32([7] * 3)
        pool = kv.K.clone()
        hb.hg_tree_masks(ctx, parents, i32(o), 64, m, d)
        hb.hg_tree_attn_paged(ctx, Q.to(DEV), i32(o), m, kv, i32(lens), 64, 60, O, L)
        hb.hg_tree_verify(ctx, tokens, parents, i32(o), 64, says, None, None, None, path, kept, nxt)
        hb.hg_tree_keep_paged(ctx, [hb.PagedKV(pool, Vp.clone(), table, 16)], i32(o), path, kept, i32(lens), 64, grown)
        torch.cuda.synchronize()
        got.append((m, d, O, L, path, kept, nxt, grown, pool.view(torch.int16)))
        ctx.close()
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert torch.isfinite(got[0][2]).all()
