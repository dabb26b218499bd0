"""Packed tokens of several sequences on the GPU: whole prompts, chunks behind a paged cache, places in it and the write there, against plain
forms in 64 bits.  Attention is held to the gates of parity.py (weights and results are rounded to bf16 as in the decode kernels), everything
else is equal bit for bit."""
import math

import numpy as np
import pytest
import torch

import oracle.fp8 as fp8
import ragged_plain as plain
from parity import check
from paper_2402_05099_amd import binding as hb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = float("nan")


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def context(mib=0):
    return hb.Context(0, mib << 20)


def rand(g, *shape, gain=1.0):
    return (torch.randn(*shape, generator=g) * gain).to(torch.bfloat16)


def verify(O, L, Oref, Lref, what, sentinel=None):
    """computed tokens pass the gates, the others are as they were"""
    done = ~torch.isnan(Lref[:, 0]) if Lref.numel() else torch.zeros(0, dtype=torch.bool)
    Oc, Lc = O.detach().cpu(), None if L is None else L.detach().cpu()
    if sentinel is not None:
        assert torch.all(Oc[~done].float() == sentinel), f"{what}: a token of nobody's was written"
        if Lc is not None:
            assert torch.all(Lc[~done] == sentinel)
    if done.any():
        check(Oc[done].double().numpy(), None if Lc is None else Lc[done].double().numpy(), Oref[done].numpy(), Lref[done].numpy(), what,
              out_bf16=O.dtype == torch.bfloat16)


def offsets(counts, lead=0):
    return np.concatenate([[lead], lead + np.cumsum(counts)]).astype(np.int64)


# ---- whole prompts -----------------------------------------------------------------------------------------------------------

def run_prompt(lens, heads, D, *, lead=0, trail=0, fused=False, fp32=False, lse=True, gain=1.0, scale=0.0, max_len=None, seed=0, mib=0, spoil=None, tilt=0.0):
    Hq, Hkv = heads
    g = torch.Generator().manual_seed(seed)
    off = offsets(lens, lead)
    T = int(off[-1]) + trail
    x = rand(g, T, Hq + 2 * Hkv, D)
    x[:, :Hq] *= gain
    if tilt:      # scores that rise along the keys, in steps of `tilt` at most
        x[:, :Hq, 0] = 1.0
        x[:, Hq:Hq + Hkv, 0] = (torch.arange(T)[:, None] * tilt * math.sqrt(D)).to(torch.bfloat16)
    x[:lead, Hq:] = NAN
    x[int(off[-1]):, Hq:] = NAN
    if spoil is not None:
        x[int(off[spoil]):int(off[spoil + 1])] = NAN
    Q, K, V = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    xd = x.to(DEV)
    Qd, Kd, Vd = xd[:, :Hq], xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:]
    if not fused:
        Qd, Kd, Vd = Qd.contiguous(), Kd.contiguous(), Vd.contiguous()
    O = torch.full((T, Hq, D), 7.0, dtype=torch.float32 if fp32 else torch.bfloat16, device=DEV)
    L = torch.full((T, Hq), 7.0, dtype=torch.float32, device=DEV) if lse else None
    ctx = context(mib)
    hb.hg_prompt_attn(ctx, Qd, Kd, Vd, i32(off), max(list(lens) + [0]) if max_len is None else max_len, O, L, scale)
    torch.cuda.synchronize()
    rows = [(int(off[b]), int(off[b + 1])) for b in range(len(lens))]
    Oref, Lref = plain.attention(Q, off, [K[a:z].double() for a, z in rows], [V[a:z].double() for a, z in rows], lens, scale or None, max_len)
    if spoil is not None:
        a, z = rows[spoil]
        keep = torch.ones(T, dtype=torch.bool)
        keep[a:z] = False
        O, Oref, Lref = O.cpu()[keep], Oref[keep], Lref[keep]
        L = None if L is None else L.cpu()[keep]
    verify(O, L, Oref, Lref, f"prompt {lens} {heads} {D}", 7.0)
    ctx.close()


HEADS = [(4, 4), (8, 1), (16, 2), (12, 4), (10, 2), (64, 8)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", HEADS)
def test_prompts_of_odd_lengths(heads, D):
    run_prompt([1, 0, 31, 32, 33, 2, 63, 64, 65, 100], heads, D, lead=5, trail=3, fused=heads[0] == 16)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [[255], [256], [257], [511, 513], [1025], [129, 300, 7, 640]])
@pytest.mark.parametrize("heads", [(4, 4), (16, 2)])
def test_longer_prompts(lens, heads, D):
    run_prompt(lens, heads, D, fused=True, mib=64)


@pytest.mark.parametrize("D", [64, 128])
def test_prompt_of_two_thousand_tokens(D):
    run_prompt([2049], (4, 2), D, fp32=True, mib=64)


def test_prompt_results_in_fp32_and_without_lse():
    run_prompt([70, 3], (8, 2), 128, fp32=True)
    run_prompt([70, 3], (8, 2), 128, lse=False)
    run_prompt([300, 3], (8, 2), 64, lse=False, scale=0.2)


def test_many_short_prompts():
    run_prompt([i % 7 for i in range(500)], (2, 1), 64)
    run_prompt([1] * 130, (16, 2), 128)


@pytest.mark.parametrize("D", [64, 128])
def test_tokens_behind_the_bound_are_left(D):
    run_prompt([300, 20, 129], (4, 2), D, max_len=128)


@pytest.mark.parametrize("gain", [4.0, 16.0])
@pytest.mark.parametrize("D", [64, 128])
def test_peaked_scores(D, gain):
    run_prompt([400, 33], (4, 2), D, gain=gain, fp32=True)


@pytest.mark.parametrize("tilt", [0.25, -0.25, 8.0])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_that_rise_and_fall_along_the_keys(D, tilt):
    run_prompt([700], (4, 2), D, tilt=tilt, fp32=True)


def test_a_sequence_of_nan_spoils_no_other():
    run_prompt([40, 65, 300, 20], (8, 2), 128, spoil=1, mib=64)
    run_prompt([40, 300, 37, 20], (8, 2), 64, spoil=1, mib=64)


def test_a_key_that_is_not_seen_yet_may_be_nan():
    g = torch.Generator().manual_seed(3)
    Q, K, V = rand(g, 300, 8, 128), rand(g, 300, 2, 128), rand(g, 300, 2, 128)
    K[290:] = NAN
    K[289] = math.inf
    O, L = torch.empty(300, 8, 128, dtype=torch.float32, device=DEV), torch.empty(300, 8, device=DEV)
    ctx = context()
    hb.hg_prompt_attn(ctx, Q.to(DEV), K.to(DEV), V.to(DEV), i32([0, 300]), 300, O, L)
    Oref, Lref = plain.attention(Q[:289], [0, 289], [K[:289]], [V[:289]], [289])
    check(O[:289].cpu().double().numpy(), L[:289].cpu().double().numpy(), Oref.numpy(), Lref.numpy(), "before the NaN")
    ctx.close()


# ---- chunks behind a paged cache ---------------------------------------------------------------------------------------------

def make_cache(g, rows_of, Hkv, D, ps, codes, scales=(0.02, 0.015), spare=2, far=0):
    """(K pool, V pool, table, keys, values): pages in a random order, rows that nobody owns are NaN, entries past a sequence's pages are wild"""
    need = [-(-r // ps) for r in rows_of]
    n_pages, stride = sum(need) + spare + far, max(need + [1])
    order = torch.randperm(sum(need) + spare, generator=g) + far
    table = torch.full((len(rows_of), stride), -7, dtype=torch.int32)
    table[:, -1:] = 1 << 30
    pool_dev = "cpu" if not far else DEV
    if codes:
        pools = [torch.full((n_pages * ps, Hkv, D), 0x7F, dtype=torch.uint8, device=pool_dev) for _ in range(2)]
    else:
        pools = [torch.full((n_pages * ps, Hkv, D), NAN, dtype=torch.bfloat16, device=pool_dev) if not far else
                 torch.empty((n_pages * ps, Hkv, D), dtype=torch.bfloat16, device=pool_dev) for _ in range(2)]
    real = [[], []]
    at = 0
    for b, r in enumerate(rows_of):
        pages = order[at:at + need[b]]
        at += need[b]
        table[b, :need[b]] = pages.int()
        j = torch.arange(r)
        where = pages[j // ps] * ps + j % ps
        for i in range(2):
            x = rand(g, r, Hkv, D)
            if codes:
                c = (x.float() / scales[i]).clamp(-448, 448).to(torch.float8_e4m3fn)
                real[i].append(c.double() * float(np.float32(scales[i])))
                x = c.view(torch.uint8)
            else:
                real[i].append(x.double())
            pools[i][where.to(pool_dev)] = x.to(pool_dev)
    return pools[0].to(DEV), pools[1].to(DEV), table.to(DEV), real[0], real[1]


def run_chunk(pairs, heads, D, *, ps=16, codes=False, lead=0, trail=0, fused=False, fp32=False, lse=True, scale=0.0, max_new=None, max_len=None, seed=0, mib=0,
              gain=1.0, far=0, ctx=None):
    """pairs: (rows in the cache with the new ones, new tokens)"""
    Hq, Hkv = heads
    g = torch.Generator().manual_seed(seed)
    lens, counts = [r for r, _ in pairs], [n for _, n in pairs]
    off = offsets(counts, lead)
    T = int(off[-1]) + trail
    scales = (0.02, 0.015)
    Kp, Vp, table, keys, values = make_cache(g, lens, Hkv, D, ps, codes, scales, far=far)
    x = rand(g, T, Hq + (3 if fused else 0), D, gain=gain)
    Q, Qd = x[:, :Hq], x.to(DEV)[:, :Hq]
    O = torch.full((T, Hq, D), 7.0, dtype=torch.float32 if fp32 else torch.bfloat16, device=DEV)
    L = torch.full((T, Hq), 7.0, dtype=torch.float32, device=DEV) if lse else None
    kv = hb.PagedKV(K=Kp, V=Vp, page_table=table, page_size=ps, kv_format=hb.HG_KV_E4M3 if codes else hb.HG_KV_BF16, k_scale=scales[0], v_scale=scales[1])
    own = ctx or context(mib)
    hb.hg_chunk_attn_paged(own, Qd, i32(off), kv, i32(lens), max(counts + [0]) if max_new is None else max_new,
                           max(lens + [0]) if max_len is None else max_len, O, L, scale)
    torch.cuda.synchronize()
    seen = lens if max_len is None else [min(r, max_len) for r in lens]
    Oref, Lref = plain.attention(Q, off, keys, values, seen, scale or None, max_new)
    verify(O, L, Oref, Lref, f"chunk {pairs[:6]} {heads} {D} {ps} {'codes' if codes else 'bf16'}", 7.0)
    if ctx is None:
        own.close()


MIXED = [(1, 1), (40, 0), (17, 17), (300, 33), (0, 0), (65, 1), (3, 5), (0, 4), (129, 64), (64, 64), (512, 2)]      # (3, 5) and (0, 4): tokens that see nothing


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", HEADS)
def test_chunks_of_every_kind(heads, D, codes):
    run_chunk(MIXED, heads, D, codes=codes, lead=2, trail=3, fused=heads[0] == 10)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ps", [16, 64, 1024])
def test_pages_of_other_sizes(ps, D, codes):
    run_chunk(MIXED, (16, 2), D, ps=ps, codes=codes, mib=64)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [(4, 4), (8, 1), (16, 2)])
@pytest.mark.parametrize("mib", [0, 64])
def test_single_tokens(heads, D, codes, mib):
    run_chunk([(r, 1) for r in (1, 2, 15, 16, 17, 31, 32, 33, 100, 255, 256, 257, 1000, 0)] + [(50, 0)], heads, D, codes=codes, mib=mib)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mib", [0, 1, 256])
def test_long_contexts_whatever_the_workspace(D, codes, mib):
    run_chunk([(9000, 1), (70, 3), (5001, 40)], (16, 2), D, ps=64, codes=codes, mib=mib, fp32=True)
    run_chunk([(9000, 1), (6000, 3)], (4, 4), D, ps=64, codes=codes, mib=mib)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_long_chunks(D, codes):
    run_chunk([(1500, 700), (801, 800), (300, 1), (2000, 257)], (8, 2), D, codes=codes, mib=256)
    run_chunk([(1111, 600)], (2, 2), D, codes=codes, ps=32, mib=256)


def test_many_single_tokens():
    run_chunk([(1 + 13 * i % 400, 1) for i in range(300)], (8, 2), 128, mib=64)
    run_chunk([(1 + 13 * i % 100, i % 3) for i in range(300)], (8, 1), 64, mib=64)


@pytest.mark.parametrize("codes", [False, True])
def test_chunk_results_in_fp32_and_without_lse(codes):
    run_chunk([(70, 3), (400, 1)], (8, 2), 128, fp32=True, codes=codes, mib=16)
    run_chunk([(70, 3), (4000, 1)], (8, 2), 128, lse=False, codes=codes, scale=0.3, mib=16)
    run_chunk([(700, 300)], (8, 2), 64, lse=False, codes=codes, scale=0.3, mib=16)


@pytest.mark.parametrize("codes", [False, True])
def test_bounds_below_the_lengths(codes):
    run_chunk([(300, 40), (90, 1), (500, 300)], (8, 2), 128, max_new=32, codes=codes)
    run_chunk([(300, 4), (90, 1), (500, 200)], (8, 2), 128, max_len=128, codes=codes)
    run_chunk([(300, 4), (90, 1)], (8, 2), 64, max_len=0, codes=codes)


@pytest.mark.parametrize("gain", [4.0, 16.0])
@pytest.mark.parametrize("D", [64, 128])
def test_peaked_scores_over_the_cache(D, gain):
    run_chunk([(900, 1), (700, 300)], (8, 2), D, gain=gain, fp32=True, mib=16)


@pytest.mark.parametrize("pairs", [[(200, 1), (90, 1)], [(700, 300)]])
def test_rows_beyond_four_gigabytes_of_pool(pairs):
    # (pages of 64 rows x 8 heads x 128: 128 KiB, the first one used 5 GiB into the pool)
    run_chunk(pairs, (16, 8), 128, ps=64, far=40960, mib=16)


def test_one_context_call_after_call():
    ctx = context(64)
    for seed in range(4):
        run_chunk([(4000, 1), (70, 3), (2001, 40 + seed)], (16, 2), 128, ps=64, mib=64, seed=seed, ctx=ctx)
    ctx.close()


def test_a_chunk_of_everything_is_a_prompt():
    g = torch.Generator().manual_seed(5)
    Q, K, V = rand(g, 333, 8, 128).to(DEV), rand(g, 333, 2, 128).to(DEV), rand(g, 333, 2, 128).to(DEV)
    off = i32([0, 100, 333])
    ctx = context(16)
    table = i32([[0, 1, 2, 3, 4, 5, 6, -1, -1, -1, -1, -1, -1, -1, -1], list(range(7, 22))])
    kv = hb.PagedKV(K=torch.zeros(22 * 16, 2, 128, dtype=torch.bfloat16, device=DEV), V=torch.zeros(22 * 16, 2, 128, dtype=torch.bfloat16, device=DEV),
                    page_table=table, page_size=16)
    hb.hg_kv_write_paged(ctx, K, V, torch.cat([torch.arange(100), torch.arange(233) + 112]).int().to(DEV), kv)
    O, L = [torch.empty(333, 8, 128, dtype=torch.float32, device=DEV) for _ in range(2)], [torch.empty(333, 8, device=DEV) for _ in range(2)]
    hb.hg_prompt_attn(ctx, Q, K, V, off, 233, O[0], L[0])
    hb.hg_chunk_attn_paged(ctx, Q, off, kv, i32([100, 233]), 233, 233, O[1], L[1])
    check(O[1].cpu().double().numpy(), L[1].cpu().double().numpy(), O[0].cpu().double().numpy(), L[0].cpu().double().numpy(), "chunk and prompt")
    ctx.close()


# ---- places in the cache -------------------------------------------------------------------------------------------------------

def run_slots(lengths, counts, ps, n_free, stride, rows=None, seed=0):
    g = np.random.default_rng(seed)
    B = len(lengths)
    table = np.full((B, stride), -1, dtype=np.int32)
    pages = g.permutation(B * stride + n_free).astype(np.int32)
    for b, x in enumerate(lengths):
        have = min(-(-max(x, 0) // ps), stride)
        table[b, :have] = pages[b * stride:b * stride + have]
    free = pages[B * stride:B * stride + n_free]
    total = sum(max(n, 0) for n in counts)
    rows = total if rows is None else rows
    want = plain.page_slots(lengths, counts, free, ps, table, rows)
    t = i32(table.tolist()) if B else torch.empty(0, stride, dtype=torch.int32, device=DEV)
    q_off, slots, new, used = (torch.full((n,), 99, dtype=torch.int32, device=DEV) for n in (B + 1, rows, B, 1))
    ctx = context()
    args = (i32(list(lengths)), i32(list(counts)), i32(free.tolist()), ps, t, q_off, slots, new, used)
    for _ in range(2):      # the second call changes nothing
        hb.hg_page_slots(ctx, *args)
        got = [x.cpu().numpy() for x in (q_off, slots, new, used, t)]
        for name, a, z in zip(("q_off", "slots", "new_lengths", "pages_used", "table"), got, want):
            assert np.array_equal(a.reshape(np.shape(z)) if name != "pages_used" else a[0], z), (name, a, z)
    ctx.close()


@pytest.mark.parametrize("ps", [16, 64, 1024])
@pytest.mark.parametrize("B", [1, 3, 64, 255, 256, 257, 700])
def test_slots_of_ragged_requests(B, ps):
    g = np.random.default_rng(B)
    run_slots(g.integers(0, 200, B).tolist(), g.integers(0, 40, B).tolist(), ps, 16 * B, 20)


def test_slots_of_long_prompts_among_single_tokens():
    run_slots([0, 17, 4000, 5, 16, 15], [9000, 1, 1, 3000, 1, 1], 16, 2000, 600)


def test_slots_at_page_borders_and_of_nobody():
    run_slots([0, 15, 16, 17, 0, 32], [16, 1, 1, 0, 0, 17], 16, 10, 4)
    run_slots([0, 0], [0, 0], 16, 0, 1)
    run_slots([], [], 16, 5, 3, rows=4)
    run_slots([-3, 5], [2, -9], 16, 5, 3)


def test_more_rows_and_fewer_than_tokens():
    run_slots([3, 40, 9], [5, 20, 700], 16, 100, 60, rows=1500)
    run_slots([3, 40, 9], [5, 20, 700], 16, 100, 60, rows=300)


def test_a_list_of_free_pages_that_is_too_short():
    run_slots([3, 40, 9, 16], [5, 20, 100, 1], 16, 4, 60)
    run_slots([3, 16, 9], [5, 20, 100], 16, 0, 60)


def test_a_table_that_is_too_narrow():
    run_slots([3, 40, 60, 64], [5, 100, 4, 3], 16, 50, 4)


# ---- the write -----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,Hkv,fused", [(1, 1, False), (45, 2, False), (333, 8, True), (70, 3, True)])
def test_rows_are_written_to_their_slots(T, Hkv, fused, D, codes):
    g = torch.Generator().manual_seed(T)
    x = rand(g, T, 2 * Hkv + (5 if fused else 0), D, gain=3.0)
    x[0, 0, :4] = torch.tensor([NAN, math.inf, -math.inf, 0.0])
    K, V = x[:, :Hkv], x[:, Hkv:2 * Hkv]
    xd = x.to(DEV)
    Kd, Vd = xd[:, :Hkv], xd[:, Hkv:2 * Hkv]
    if not fused:
        Kd, Vd = Kd.contiguous(), Vd.contiguous()
    pages = -(-T // 16) + 3
    slots = torch.randperm(pages * 16, generator=g)[:T].int()
    if T > 8:
        slots[3], slots[5], slots[6] = -1, pages * 16, -(1 << 31)
    dt = torch.uint8 if codes else torch.bfloat16
    pools = [torch.full((pages * 16, Hkv, D), 5, dtype=dt) for _ in range(2)]
    dev = [p.to(DEV) for p in pools]
    scales = (0.01, 0.03)
    kv = hb.PagedKV(K=dev[0], V=dev[1], page_table=i32([[0]]), page_size=16, kv_format=int(codes), k_scale=scales[0], v_scale=scales[1])
    ctx = context()
    hb.hg_kv_write_paged(ctx, Kd, Vd, slots.to(DEV), kv)
    ok = (slots >= 0) & (slots < pages * 16)
    for pool, got, new, scale in zip(pools, dev, (K, V), scales):
        if codes:
            new = torch.from_numpy(fp8.quantize(new.float().numpy(), np.float32(scale)))
        pool[slots[ok].long()] = new[ok]
        a, z = (pool, got.cpu()) if codes else (pool.view(torch.int16), got.cpu().view(torch.int16))
        assert torch.equal(a, z)
    ctx.close()


# ---- streams, graphs, refusals ---------------------------------------------------------------------------------------------------

def test_a_captured_step_follows_its_lengths():
    """slots, write and chunk attention in one graph, replayed with other lengths in the same tensors, equal the eager calls each time"""
    g = torch.Generator().manual_seed(11)
    B, Hq, Hkv, D, ps, stride, T = 5, 16, 2, 128, 16, 40, 256
    table = torch.full((B, stride), -1, dtype=torch.int32, device=DEV)
    pool = [torch.zeros(400 * ps, Hkv, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    kv = hb.PagedKV(K=pool[0], V=pool[1], page_table=table, page_size=ps)
    lengths, counts, free = i32([0] * B), i32([0] * B), torch.randperm(400, generator=g).int().to(DEV)
    q_off, slots, new, used = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in (B + 1, T, B, 1))
    x = rand(g, T, Hq + 2 * Hkv, D).to(DEV)
    Q, K, V = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    O, L = torch.zeros(T, Hq, D, dtype=torch.bfloat16, device=DEV), torch.zeros(T, Hq, device=DEV)
    stream = torch.cuda.Stream()
    ctx = hb.Context(0, 64 << 20, stream=stream)

    def step():
        hb.hg_page_slots(ctx, lengths, counts, free, ps, table, q_off, slots, new, used)
        hb.hg_kv_write_paged(ctx, K, V, slots, kv)
        hb.hg_chunk_attn_paged(ctx, Q, q_off, kv, new, 128, stride * ps, O, L)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for n in ([10, 0, 128, 1, 33], [1, 1, 1, 1, 1], [0, 100, 0, 0, 0], [50, 3, 2, 1, 128]):
        counts.copy_(i32(n))
        for t in (*pool, O, L):
            t.zero_()
        table.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (table, q_off, slots, new, used, *pool, O, L)]
        for t in (*pool, O, L):
            t.zero_()
        table.fill_(-1)
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        for a, z in zip(got, (table, q_off, slots, new, used, *pool, O, L)):
            assert torch.equal(a, z)
        off = np.concatenate([[0], np.cumsum(n)])
        Oref, Lref = plain.attention(Q.cpu(), off, [K[a:z].cpu().double() for a, z in zip(off, off[1:])], [V[a:z].cpu().double() for a, z in zip(off, off[1:])], n)
        done = ~torch.isnan(Lref[:, 0])
        check(O.cpu()[done].double().numpy(), L.cpu()[done].double().numpy(), Oref[done].numpy(), Lref[done].numpy(), f"step {n}", out_bf16=True)
    ctx.close()


def test_refusals_leave_everything_as_it_was():
    ctx = context()
    bf, f32 = dict(dtype=torch.bfloat16, device=DEV), dict(dtype=torch.float32, device=DEV)
    Q, K, V, O, L = torch.zeros(8, 4, 64, **bf), torch.zeros(8, 2, 64, **bf), torch.zeros(8, 2, 64, **bf), torch.full((8, 4, 64), 7.0, **bf), torch.full((8, 4), 7.0, **f32)
    off = i32([0, 8])
    pool = torch.zeros(32, 2, 64, **bf)
    kv = hb.PagedKV(K=pool, V=pool.clone(), page_table=i32([[0, 1]]), page_size=16)
    bad = lambda **k: hb.PagedKV(**{**dict(K=kv.K, V=kv.V, page_table=kv.page_table, page_size=16), **k})  # noqa: E731
    eight = dict(K=torch.zeros(32, 2, 64, dtype=torch.uint8, device=DEV), V=torch.zeros(32, 2, 64, dtype=torch.uint8, device=DEV), kv_format=hb.HG_KV_E4M3)
    wide = torch.zeros(8, 4, 132, **bf)
    calls = [
        (TypeError, lambda: hb.hg_prompt_attn(ctx, Q.float(), K, V, off, 8, O, L)),
        (TypeError, lambda: hb.hg_prompt_attn(ctx, Q, K.cpu(), V, off, 8, O, L)),
        (TypeError, lambda: hb.hg_prompt_attn(ctx, Q, K, V, off.long(), 8, O, L)),
        (ValueError, lambda: hb.hg_prompt_attn(ctx, Q, K, V[:7], off, 8, O, L)),
        (ValueError, lambda: hb.hg_prompt_attn(ctx, wide[:, :, :64], K, V, off, 8, O, L)),
        (ValueError, lambda: hb.hg_prompt_attn(ctx, Q, K, V, off, 8, O[:4], L)),
        (hb.HG_ERR_UNSUPPORTED, lambda: hb.hg_prompt_attn(ctx, torch.zeros(8, 3, 64, **bf), K, V, off, 8, torch.zeros(8, 3, 64, **bf))),
        (hb.HG_ERR_UNSUPPORTED, lambda: hb.hg_prompt_attn(ctx, torch.zeros(8, 4, 32, **bf), torch.zeros(8, 2, 32, **bf), torch.zeros(8, 2, 32, **bf), off, 8, torch.zeros(8, 4, 32, **bf))),
        (hb.HG_ERR_INVALID_ARG, lambda: hb.hg_prompt_attn(ctx, Q, K, V, off, -1, O, L)),
        (hb.HG_ERR_INVALID_ARG, lambda: hb.hg_chunk_attn_paged(ctx, Q, off, kv, i32([8]), 8, 33, O, L)),
        (hb.HG_ERR_INVALID_ARG, lambda: hb.hg_chunk_attn_paged(ctx, Q, off, kv, i32([8]), -1, 8, O, L)),
        (hb.HG_ERR_INVALID_ARG, lambda: hb.hg_chunk_attn_paged(ctx, Q, off, bad(**eight, k_scale=0.0), i32([8]), 8, 8, O, L)),
        (hb.HG_ERR_INVALID_ARG, lambda: hb.hg_chunk_attn_paged(ctx, Q, off, bad(**eight, v_scale=math.inf), i32([8]), 8, 8, O, L)),
        (hb.HG_ERR_INVALID_ARG, lambda: hb.hg_chunk_attn_paged(ctx, Q, off, bad(page_size=8), i32([8]), 8, 8, O, L)),
        (ValueError, lambda: hb.hg_chunk_attn_paged(ctx, Q, i32([0, 4, 8]), kv, i32([4, 4]), 8, 8, O, L)),
        (ValueError, lambda: hb.hg_chunk_attn_paged(ctx, Q, off, kv, i32([4, 4]), 8, 8, O, L)),
        (hb.HG_ERR_INVALID_ARG, lambda: hb.hg_page_slots(ctx, i32([0]), i32([1]), i32([0]), 24, i32([[0]]), i32([0, 0]), i32([0]), i32([0]), i32([0]))),
        (ValueError, lambda: hb.hg_page_slots(ctx, i32([0]), i32([1, 2]), i32([0]), 16, i32([[0]]), i32([0, 0]), i32([0]), i32([0]), i32([0]))),
        (TypeError, lambda: hb.hg_kv_write_paged(ctx, K, V, i32([0] * 8), bad(**eight, page_size=16).__class__(**{**vars(kv), "kv_format": hb.HG_KV_E4M3}))),
        (hb.HG_ERR_INVALID_ARG, lambda: hb.hg_kv_write_paged(ctx, K, V, i32([0] * 8), bad(**eight, k_scale=-1.0))),
        (ValueError, lambda: hb.hg_kv_write_paged(ctx, K, V, i32([0] * 7), kv)),
    ]
    same = i32([0])
    calls.append((hb.HG_ERR_INVALID_ARG, lambda: hb.hg_page_slots(ctx, same, i32([1]), i32([0]), 16, i32([[0]]), i32([0, 0]), i32([0]), same, i32([0]))))
    for i, (what, call) in enumerate(calls):
        if isinstance(what, int):
            with pytest.raises(hb.HydragenError) as e:
                call()
            assert e.value.code == what, i
        else:
            with pytest.raises(what):
                call()
    torch.cuda.synchronize()
    assert torch.all(O.float() == 7.0) and torch.all(L == 7.0) and torch.all(pool == 0)
    ctx.close()


def test_nothing_to_do_is_fine():
    ctx = context()
    bf = dict(dtype=torch.bfloat16, device=DEV)
    e = torch.zeros(0, 4, 64, **bf)
    kv = hb.PagedKV(K=torch.zeros(16, 4, 64, **bf), V=torch.zeros(16, 4, 64, **bf), page_table=i32([[0]]), page_size=16)
    hb.hg_prompt_attn(ctx, e, e, e, i32([0, 0]), 5, e.clone())
    hb.hg_prompt_attn(ctx, e, e, e, i32([0]), 5, e.clone())
    hb.hg_chunk_attn_paged(ctx, e, i32([0, 0]), kv, i32([3]), 1, 16, e.clone())
    hb.hg_kv_write_paged(ctx, e, e, torch.zeros(0, dtype=torch.int32, device=DEV), kv)
    torch.cuda.synchronize()
    ctx.close()


def test_same_results_through_the_checks_in_python(monkeypatch):
    """the native marshalling and the checks in Python make the same calls"""
    calls = []
    for native in (hb.native(), hb._PythonOnly):
        monkeypatch.setattr(hb, "_native", native)
        run_prompt([40, 3, 200], (8, 2), 128, fused=True, lse=False)
        run_chunk([(300, 33), (65, 1), (3, 5)], (8, 2), 64, codes=True, fused=True, mib=16)
        run_slots([3, 40, 9], [5, 20, 100], 16, 60, 60)
        calls.append(native)
    assert len(calls) == 2
    m = hb.native() if hb._native is not hb._PythonOnly else calls[0]
    q = torch.zeros(2, 2, 64, dtype=torch.bfloat16)      # host tensors: left to Python
    assert m.prompt(None, q, q, q, q, 1, q, q, 0.0) is None and m.chunk(*[object()] * 10) is None
    assert m.slots() is None and m.write(1, 2, 3, 4, 5) is None


# ---- where tiles end and what remains begins ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_every_kind_of_remainder(D, codes):
    # one row a token: 128-row tiles, and behind them 0, 1, 16, 17, 32, 33, 64 (few rows) or 65, 127 rows (a tile)
    for counts in ([64, 65, 127, 128, 129], [144, 145, 160, 161, 192, 193, 255, 256, 257]):
        run_chunk([(n + 37 * i, n) for i, n in enumerate(counts)], (2, 2), D, codes=codes, mib=16)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("heads", [(80, 1), (64, 1), (9, 3), (14, 2)])
def test_groups_of_heads_of_every_size(heads, codes):
    run_chunk([(100, 1), (90, 2), (77, 3), (200, 40), (5, 0)], heads, 64, codes=codes, mib=16)
    if not codes:
        run_prompt([1, 2, 3, 30, 70], heads, 64)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_tokens_of_long_chunks_that_see_nothing(D, codes):
    run_chunk([(200, 300), (0, 200), (100, 400), (1, 130)], (2, 2), D, codes=codes, mib=16)
    run_chunk([(5, 200), (300, 290)], (8, 2), D, codes=codes, fp32=True)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("B", [8, 9, 64, 65, 150])
def test_long_chunks_among_many_sequences(B, codes):
    run_chunk([(40 + 7 * i % 90 + n, n) for i, n in ((i, (1, 0, 150, 1, 70, 1, 1, 33)[i % 8]) for i in range(B))], (4, 2), 64, codes=codes, mib=16, lead=1)
    if not codes:
        run_prompt([(1, 0, 150, 3, 70)[i % 5] for i in range(B)], (4, 2), 64, lead=3, trail=2)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_tiles_of_long_contexts_are_split(D, codes):
    run_chunk([(17000, 140)], (2, 2), D, codes=codes, mib=256, ps=64)
    run_chunk([(9000, 130), (12000, 1), (300, 200), (2048, 64)], (4, 2), D, codes=codes, mib=256, ps=64, fp32=True)
    run_chunk([(9000, 130), (12000, 1)], (4, 2), D, codes=codes, mib=256, ps=64, lse=False)


def test_a_long_prompt_of_one_head_is_split():
    run_prompt([5000], (1, 1), 128, mib=256)
    run_prompt([4000, 17], (1, 1), 64, mib=256, fp32=True)


def test_the_same_call_gives_the_same_bits():
    g = torch.Generator().manual_seed(2)
    pairs = [(5000, 140), (9000, 1), (300, 33)]
    Kp, Vp, table, _, _ = make_cache(g, [r for r, _ in pairs], 2, 128, 64, False)
    off = offsets([n for _, n in pairs])
    Q = rand(g, int(off[-1]), 8, 128).to(DEV)
    kv = hb.PagedKV(K=Kp, V=Vp, page_table=table, page_size=64)
    ctx = context(64)
    got = []
    for _ in range(3):
        O, L = torch.empty(int(off[-1]), 8, 128, device=DEV), torch.empty(int(off[-1]), 8, device=DEV)
        hb.hg_chunk_attn_paged(ctx, Q, i32(off), kv, i32([r for r, _ in pairs]), 140, 9000, O, L)
        got.append((O.clone(), L.clone()))
    assert all(torch.equal(a, b) for g_ in got[1:] for a, b in zip(g_, got[0]))
    ctx.close()


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B", [30, 40])      # 120 columns of 64 rows at most are a small call, 160 are not
def test_calls_of_up_to_sixty_four_rows(B, D, codes):
    pairs = [(3 + 29 * i % 500, (9, 16, 1, 12, 0, 8)[i % 6]) for i in range(B)]
    run_chunk(pairs, (16, 4), D, codes=codes, mib=16)
    run_chunk(pairs, (16, 4), D, codes=codes, fp32=True, lead=1)
    run_chunk([(3000, 16), (1, 16)] + pairs, (16, 4), D, codes=codes, mib=64, ps=64)


# ---- values that are infinite or NaN reach the tokens that see them, and no others -----------------------------------------------------

BAD = [(math.nan, 3), (math.inf, 17), (-math.inf, 40), (math.nan, 63)]      # value, column


def with_bad_values(run, O, L, Oref, Lref, off, lens, counts, spoiled, G, what):
    """spoiled: (sequence, key, KV head, column, value); Oref was taken with zeros in their places"""
    run()
    torch.cuda.synchronize()
    O, L = O.cpu().double(), L.cpu().double()
    got_all = O.clone()
    assert torch.isfinite(Oref).all()
    for b, key, h, d, x in spoiled:
        for t in range(counts[b]):
            if key < lens[b] - (counts[b] - 1 - t):
                got = got_all[int(off[b]) + t, h * G:(h + 1) * G, d]
                assert not torch.isfinite(got).any(), f"{what}: token {t} of {b} sees {x} in row {key} and does not show it"
                O[int(off[b]) + t, h * G:(h + 1) * G, d] = Oref[int(off[b]) + t, h * G:(h + 1) * G, d]
    check(O.numpy(), L.numpy(), Oref.numpy(), Lref.numpy(), what)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [(2, 2), (8, 2), (16, 1)])
def test_values_that_are_not_seen_yet_may_be_anything(heads, D):
    Hq, Hkv = heads
    G = Hq // Hkv
    lens = [300, 1, 77, 140, 33]
    off = offsets(lens)
    g = torch.Generator().manual_seed(D + Hq)
    T = int(off[-1])
    Q, K, V = rand(g, T, Hq, D), rand(g, T, Hkv, D), rand(g, T, Hkv, D)
    spoiled = [(b, key, i % Hkv, BAD[i % 4][1], BAD[i % 4][0]) for i, (b, key) in
               enumerate([(0, 5), (0, 100), (0, 131), (0, 255), (0, 256), (0, 299), (2, 40), (2, 76), (3, 127), (3, 128), (4, 31), (4, 32)])]
    bad = V.clone()
    for b, key, h, d, x in spoiled:
        V[int(off[b]) + key, h, d] = 0
        bad[int(off[b]) + key, h, d] = x
    rows = [(int(off[b]), int(off[b + 1])) for b in range(len(lens))]
    Oref, Lref = plain.attention(Q, off, [K[a:z].double() for a, z in rows], [V[a:z].double() for a, z in rows], lens)
    O, L = torch.empty(T, Hq, D, device=DEV), torch.empty(T, Hq, device=DEV)
    ctx = context()
    with_bad_values(lambda: hb.hg_prompt_attn(ctx, Q.to(DEV), K.to(DEV), bad.to(DEV), i32(off), max(lens), O, L), O, L, Oref, Lref, off, lens, lens, spoiled, G,
                    f"prompts {heads} {D}")
    ctx.close()


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [(2, 2), (8, 2), (16, 1)])
def test_values_of_later_tokens_in_the_cache_may_be_anything(heads, D, codes):
    Hq, Hkv = heads
    G = Hq // Hkv
    ps, scales = 32, (0.02, 0.015)
    pairs = [(200, 3), (90, 1), (300, 150), (64, 64), (2000, 9), (33, 2)]
    lens, counts = [r for r, _ in pairs], [n for _, n in pairs]
    off = offsets(counts)
    g = torch.Generator().manual_seed(D + Hq)
    Kp, Vp, table, keys, values = make_cache(g, lens, Hkv, D, ps, codes, scales)
    spoiled = [(b, key, i % Hkv, BAD[i % 4][1], BAD[i % 4][0]) for i, (b, key) in
               enumerate([(0, 198), (0, 199), (2, 160), (2, 191), (2, 230), (2, 299), (3, 0), (3, 31), (3, 63), (4, 1992), (4, 1999), (5, 32)])]
    for b, key, h, d, x in spoiled:
        values[b][key, h, d] = 0
        row = int(table[b, key // ps]) * ps + key % ps
        Vp[row, h, d] = (0x7F if x > 0 else 0xFF) if codes else x
    Q = rand(g, int(off[-1]), Hq, D)
    Oref, Lref = plain.attention(Q, off, keys, values, lens)
    kv = hb.PagedKV(K=Kp, V=Vp, page_table=table, page_size=ps, kv_format=hb.HG_KV_E4M3 if codes else hb.HG_KV_BF16, k_scale=scales[0], v_scale=scales[1])
    O, L = torch.empty(int(off[-1]), Hq, D, device=DEV), torch.empty(int(off[-1]), Hq, device=DEV)
    for mib in (0, 64):
        ctx = context(mib)
        with_bad_values(lambda: hb.hg_chunk_attn_paged(ctx, Q.to(DEV), i32(off), kv, i32(lens), max(counts), max(lens), O, L), O, L, Oref, Lref, off, lens, counts,
                        spoiled, G, f"chunks {heads} {D} {'codes' if codes else 'bf16'} {mib}")
        ctx.close()
    # few rows alone
    few = [0, 1, 4, 5]
    qo, ln, ct = offsets([counts[b] for b in few]), [lens[b] for b in few], [counts[b] for b in few]
    Qf = torch.cat([Q[int(off[b]):int(off[b + 1])] for b in few])
    kv = hb.PagedKV(K=Kp, V=Vp, page_table=table[few].contiguous(), page_size=ps, kv_format=kv.kv_format, k_scale=scales[0], v_scale=scales[1])
    O, L = torch.empty(int(qo[-1]), Hq, D, device=DEV), torch.empty(int(qo[-1]), Hq, device=DEV)
    ctx = context(64)
    Oref, Lref = plain.attention(Qf, qo, [keys[b] for b in few], [values[b] for b in few], ln)
    with_bad_values(lambda: hb.hg_chunk_attn_paged(ctx, Qf.to(DEV), i32(qo), kv, i32(ln), max(ct), max(ln), O, L), O, L, Oref, Lref, qo, ln, ct,
                    [(few.index(b), *rest) for b, *rest in spoiled if b in few], G, f"few rows {heads} {D} {'codes' if codes else 'bf16'}")
    ctx.close()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("where", ["query", "key"])
def test_a_token_that_meets_a_nan_says_so(D, where):
    lens = [200, 40]
    off, g = offsets(lens), torch.Generator().manual_seed(D)
    Q, K, V = rand(g, 240, 4, D), rand(g, 240, 2, D), rand(g, 240, 2, D)
    rows = [(0, 200), (200, 240)]
    Oref, Lref = plain.attention(Q, off, [K[a:z].double() for a, z in rows], [V[a:z].double() for a, z in rows], lens)
    if where == "query":
        lost = torch.tensor([3, 150, 239])
        Q[lost] = NAN
    else:
        lost = torch.arange(100, 200)
        K[100] = NAN
    kept = torch.ones(240, dtype=torch.bool)
    kept[lost] = False
    O, L = torch.empty(240, 4, D, device=DEV), torch.empty(240, 4, device=DEV)
    ctx = context()
    hb.hg_prompt_attn(ctx, Q.to(DEV), K.to(DEV), V.to(DEV), i32(off), 200, O, L)
    O, L = O.cpu().double(), L.cpu().double()
    assert torch.isnan(O[~kept]).all() and torch.isnan(L[~kept]).all()
    check(O[kept].numpy(), L[kept].numpy(), Oref[kept].numpy(), Lref[kept].numpy(), f"prompt with a NaN {where}")
    ctx.close()


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("where", ["query", "key"])
@pytest.mark.parametrize("mib", [0, 64])
def test_a_token_that_meets_a_nan_in_the_cache_says_so(mib, where, D, codes):
    for pairs in ([(5000, 1), (300, 6), (40, 1)], [(5000, 150), (300, 6), (40, 1)]):
        lens, counts = [r for r, _ in pairs], [n for _, n in pairs]
        off, g = offsets(counts), torch.Generator().manual_seed(D)
        Kp, Vp, table, keys, values = make_cache(g, lens, 2, D, 64, codes)
        T = int(off[-1])
        Q = rand(g, T, 4, D)
        Oref, Lref = plain.attention(Q, off, keys, values, lens)
        if where == "query":
            lost = torch.tensor([0, int(off[1]) + 2, T - 1])
            Q[lost] = NAN
        else:      # one that all tokens of two sequences see
            lost = torch.cat([torch.arange(0, counts[0]), torch.arange(int(off[1]), int(off[2]))])
            for b, j in ((0, 3000), (1, 70)):
                Kp[int(table[b, j // 64]) * 64 + j % 64] = 0x7F if codes else NAN
        kept = torch.ones(T, dtype=torch.bool)
        kept[lost] = False
        kv = hb.PagedKV(K=Kp, V=Vp, page_table=table, page_size=64, kv_format=hb.HG_KV_E4M3 if codes else hb.HG_KV_BF16, k_scale=0.02, v_scale=0.015)
        O, L = torch.empty(T, 4, D, device=DEV), torch.empty(T, 4, device=DEV)
        ctx = context(mib)
        hb.hg_chunk_attn_paged(ctx, Q.to(DEV), i32(off), kv, i32(lens), max(counts), max(lens), O, L)
        O, L = O.cpu().double(), L.cpu().double()
        assert torch.isnan(O[~kept]).all() and torch.isnan(L[~kept]).all()
        check(O[kept].numpy(), L[kept].numpy(), Oref[kept].numpy(), Lref[kept].numpy(), f"chunks with a NaN {where}")
        ctx.close()
