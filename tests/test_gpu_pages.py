"""Block tables, slots and the write into a paged cache: refusals, the checks in Python, calls of many sequences, a list of free pages that is too short."""
import numpy as np
import pytest
import torch

from paper_2402_05099_amd import binding as hb
from test_gpu_ragged import DEV, context, i32

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
