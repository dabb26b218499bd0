"""Block tables, slots and the write into a paged cache: refusals, the checks in Python, calls of many sequences, a list of free pages that is too short."""
import numpy as np
import numpy as np
import pytest
import torch

import oracle.fp8 as fp8
import ragged_plain as plain
from parity import check
from paper_2402_05099_amd import binding as hb
from test_gpu_ragged import DEV, context, i32, rand, run_slots

pytestmark = pytest.mark.gpu


def test_a_pool_that_ends_inside_a_page_is_refused():
    """as in the calls that read it: rows behind the last whole page have no slot, and would be dropped"""
    ctx = context()
    pool = torch.full((40, 2, 64), 5, dtype=torch.uint8, device=DEV)
    for dt, fmt in ((torch.bfloat16, hb.HG_KV_BF16), (torch.uint8, hb.HG_KV_E4M3)):
        K, V = (pool.to(dt).clone() for _ in range(2))
        kv = hb.PagedKV(K=K, V=V, page_table=i32([[0, 1]]), page_size=16, kv_format=fmt)
        new = torch.ones(3, 2, 64, dtype=torch.bfloat16, device=DEV)
        with pytest.raises(ValueError, match="n_pages"):
            hb.hg_kv_write_paged(ctx, new, new, i32([0, 31, 35]), kv)
        with pytest.raises(ValueError, match="n_pages"):
            hb.hg_chunk_attn_paged(ctx, new, i32([0, 3]), kv, i32([3]), 3, 3, new.clone())
        torch.cuda.synchronize()
        assert torch.all(K == 5) and torch.all(V == 5)
    ctx.close()


@pytest.mark.parametrize("ps", [16, 128])
@pytest.mark.parametrize("B", [1023, 1024, 1025, 2048, 2049, 2500])
def test_slots_of_more_requests_than_a_pass_looks_at(B, ps):
    print(f"slots: B {B}, page {ps}", flush=True)
    g = np.random.default_rng(B)
    lengths, counts = g.integers(0, 300, B).tolist(), g.integers(0, 12, B).tolist()
    run_slots(lengths, counts, ps, 2 * B, 24)
    run_slots(lengths, counts, ps, B // 40, 24)                          # the list ends in the first pass
    run_slots(lengths, [0] * (B - 20) + [700] * 20, ps, 1000, 24)         # ... or in the last; tables too narrow for some
    run_slots(lengths, counts, ps, 2 * B, 24, rows=sum(counts[:900]))    # tokens without a place in `slots`, in every pass but the first
    run_slots(lengths, counts, ps, 2 * B, 24, rows=sum(counts) + 3000)
    run_slots([0] * B, [1] + [0] * (B - 2) + [40], ps, 5, 24)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_the_write_is_the_same_through_the_checks_in_python(D, codes, monkeypatch):
    T, Hkv, pages, scales = 77, 3, 9, (0.01, 0.03)
    g = torch.Generator().manual_seed(D)
    x = rand(g, T, 2 * Hkv + 4, D, gain=3.0)
    x[0, 1, :3] = torch.tensor([float("nan"), float("inf"), -float("inf")])
    xd = x.to(DEV)
    K, V = xd[:, 1:1 + Hkv], xd[:, 1 + Hkv:1 + 2 * Hkv]      # rows lie further apart than they are long
    assert K.stride(0) > Hkv * D
    slots = torch.randperm(pages * 16, generator=g)[:T].int()
    slots[5], slots[9] = -1, pages * 16
    ok = (slots >= 0) & (slots < pages * 16)
    dt = torch.uint8 if codes else torch.bfloat16
    want = []
    for first, scale in ((1, scales[0]), (1 + Hkv, scales[1])):
        new, pool = x[:, first:first + Hkv], torch.full((pages * 16, Hkv, D), 5, dtype=dt)
        if codes:
            new = torch.from_numpy(fp8.quantize(new.float().numpy(), np.float32(scale)))
        pool[slots[ok].long()] = new[ok]
        want.append(pool)
    ctx = context()
    for native in (hb.native(), hb._PythonOnly):
        monkeypatch.setattr(hb, "_native", native)
        pools = [torch.full((pages * 16, Hkv, D), 5, dtype=dt, device=DEV) for _ in range(2)]
        kv = hb.PagedKV(K=pools[0], V=pools[1], page_table=i32([[0]]), page_size=16, kv_format=int(codes), k_scale=scales[0], v_scale=scales[1])
        hb.hg_kv_write_paged(ctx, K, V, slots.to(DEV), kv)
        for a, z in zip(want, pools):
            a, z = (a, z.cpu()) if codes else (a.view(torch.int16), z.cpu().view(torch.int16))
            assert torch.equal(a, z), native
    ctx.close()


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("codes", [False, True])
def test_a_step_that_ran_out_of_pages_is_made_again(codes, captured):
    """slots, write and attention one after another: sequences whose tokens all have a place are right, and made again with a longer list all are"""
    g = torch.Generator().manual_seed(3)
    Hq, Hkv, D, ps, stride, counts, scales = 8, 2, 128, 16, 8, [20, 0, 70, 1, 40], (0.0125, 0.0125)
    T, B = sum(counts), len(counts)
    off = np.concatenate([[0], np.cumsum(counts)])
    x = rand(g, T, Hq + 2 * Hkv, D)
    xd = x.to(DEV)
    dt = torch.uint8 if codes else torch.bfloat16
    kv = hb.PagedKV(K=torch.zeros(20 * ps, Hkv, D, dtype=dt, device=DEV), V=torch.zeros(20 * ps, Hkv, D, dtype=dt, device=DEV),
                    page_table=torch.full((B, stride), -1, dtype=torch.int32, device=DEV), page_size=ps, kv_format=int(codes), k_scale=scales[0], v_scale=scales[1])
    pages = torch.randperm(20, generator=g).int().to(DEV)
    lengths, n = i32([0] * B), i32(counts)
    q_off, slots, new, used = (torch.zeros(k, dtype=torch.int32, device=DEV) for k in (B + 1, T, B, 1))
    O, L = torch.zeros(T, Hq, D, dtype=torch.bfloat16, device=DEV), torch.zeros(T, Hq, device=DEV)
    stream = torch.cuda.Stream()
    ctx = hb.Context(0, 16 << 20, stream=stream)

    def step(free):
        hb.hg_page_slots(ctx, lengths, n, free, ps, kv.page_table, q_off, slots, new, used)
        hb.hg_kv_write_paged(ctx, xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:], slots, kv)
        hb.hg_chunk_attn_paged(ctx, xd[:, :Hq], q_off, kv, new, 70, stride * ps, O, L)

    def stored(v):
        return (v.float() / np.float32(0.0125)).clamp(-448, 448).to(torch.float8_e4m3fn).double() * float(np.float32(0.0125)) if codes else v.double()

    K, V = ([stored(x[a:z, h:h + Hkv]) for a, z in zip(off, off[1:])] for h in (Hq, Hq + Hkv))
    Oref, Lref = plain.attention(x[:, :Hq], off, K, V, counts)
    for n_free, right in ((8, (0, 2, 3)), (11, (0, 2, 3, 4))):      # 2 + 5 + 1 + 3 pages are wanted
        free = pages[:n_free].contiguous()
        torch.cuda.synchronize()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                step(free)
            torch.cuda.synchronize()
            for _ in range(3):
                graph.replay()
        else:
            step(free)
        torch.cuda.synchronize()
        assert used.item() == 11 and lengths.tolist() == [0] * B and q_off.tolist() == off.tolist()
        assert [b for b in range(B) if new[b] == counts[b] > 0] == list(right)
        at = torch.cat([torch.arange(off[b], off[b + 1]) for b in right])
        check(O.cpu()[at].double().numpy(), L.cpu()[at].double().numpy(), Oref[at].numpy(), Lref[at].numpy(), f"{n_free} pages", out_bf16=True)
    ctx.close()
