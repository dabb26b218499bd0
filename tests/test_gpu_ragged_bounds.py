"""Calls between a prompt and its first decode step whose host bounds are a capacity, or none at all, instead of the batch's own maximum, and batches of more
sequences than 64 * 64, which are looked through in three levels."""
import pytest
import torch

import test_gpu_ragged
from test_gpu_ragged import run_chunk, run_prompt

pytestmark = pytest.mark.gpu
NO_BOUND = 2**31 - 1


@pytest.mark.parametrize("mib", [0, 1, 512])
@pytest.mark.parametrize("bound", [8192, 1 << 20, 1 << 30, NO_BOUND - 1, NO_BOUND])
def test_prompts_under_a_bound_beyond_their_tokens(bound, mib):
    print(f"prompts, bound {bound}, workspace {mib} MiB", flush=True)
    run_prompt([100, 28], (4, 4), 64, max_len=bound, mib=mib)
    run_prompt([1, 0, 64, 17], (4, 4), 128, max_len=bound, mib=mib)
    run_prompt([3000, 40], (2, 1), 128, max_len=bound, mib=mib, fp32=True)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("max_new,max_len", [(None, 4096), (None, 32768), (8, 32768), (300, 8192)])
def test_chunks_under_a_capacity(max_new, max_len, codes, monkeypatch):
    """a table for max_len rows; with a workspace there are key ranges for contexts that nobody has"""
    make_cache = test_gpu_ragged.make_cache

    def wide(*args, **more):      # entries behind a request's pages are wild
        Kp, Vp, table, keys, values = make_cache(*args, **more)
        return Kp, Vp, torch.cat([table, torch.full((table.shape[0], max_len // 16), -9, dtype=torch.int32, device=table.device)], 1), keys, values

    monkeypatch.setattr(test_gpu_ragged, "make_cache", wide)
    pairs = [(1 + 29 * i % 515, (1, 3, 0, 8)[i % 4] if max_new else 1) for i in range(45)]
    for D, mib in ((128, 64), (64, 64), (128, 0)):
        print(f"chunks, D {D}, max_new {max_new}, max_len {max_len}, workspace {mib} MiB", flush=True)
        run_chunk(pairs, (16, 2), D, codes=codes, max_new=max_new, max_len=max_len, mib=mib)


@pytest.mark.parametrize("B", [4096, 4097, 5000, 9000])
def test_very_many_sequences(B):
    print(f"prompts and chunks, B {B}", flush=True)
    few = {0: 3, 63: 140, 64: 1, 4095: 70, B // 2: 129, B - 2: 200, B - 1: 5}
    counts = [few.get(i, 0) for i in range(B)]
    run_prompt(counts, (2, 1), 64, lead=2, trail=3, mib=16)
    # key ranges, of tiles and of what remains, that are joined
    run_chunk([(n + (3000 if i in (63, B // 2, B - 1) else i % 5), n) for i, n in enumerate(counts)], (2, 1), 64, mib=256, lead=1)
    run_chunk([(1 + i % 3, 1) for i in range(B)], (2, 1), 64, mib=16)
