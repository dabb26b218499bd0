#!/usr/bin/env python3
"""One attention layer of a server that admits prompts into a running batch, behind a system prompt that all requests share.

Every step is the same five calls, whatever the requests bring (whole prompts, the next piece of one, single tokens, nothing):

  hg_page_slots        places for the new tokens in the page pool, from the lengths and counts that lie on the GPU
  hg_kv_write_paged    their K and V rows to those places
  hg_chunk_attn_paged  each token's attention over its own request's rows
  hg_prefix_attn       ... and over the system prompt, which is stored once: all tokens of all requests in one matrix
  hg_merge             the two parts into the exact result

The system prompt itself is a prompt like any other: hg_prompt_attn.  Nothing is read back between the calls; the host looks once a step, to know
how many pages of its free list are gone and whether every token had a place.

usage: prompts_to_decode.py [--requests N] [--steps K] [--system P] [--heads 32/8] [--dim 128] [--codes]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2402_05099_amd import binding as hb  # noqa: E402


class Server:
    """The pool, the block table and the lengths of `requests` requests of one layer, and the step."""

    def __init__(self, requests, heads, dim, system_k, system_v, pages, page_size=16, row_capacity=4096, codes=False, most_tokens=8192, device="cuda:0"):
        self.Hq, self.Hkv = heads
        self.D, self.page_size, self.B = dim, page_size, requests
        i32 = dict(dtype=torch.int32, device=device)
        dtype = torch.uint8 if codes else torch.bfloat16
        pool = [torch.zeros(pages * page_size, self.Hkv, dim, dtype=dtype, device=device) for _ in range(2)]
        self.kv = hb.PagedKV(K=pool[0], V=pool[1], page_table=torch.full((requests, row_capacity // page_size), -1, **i32), page_size=page_size,
                             kv_format=hb.HG_KV_E4M3 if codes else hb.HG_KV_BF16, k_scale=0.0125, v_scale=0.0125)
        self.row_capacity = row_capacity
        self.system = system_k, system_v                 # [P, Hkv, D], stored once
        self.free = torch.arange(pages, **i32)           # pages that nobody has, handed out from the front
        self.lengths, self.grown = torch.zeros(requests, **i32), torch.zeros(requests, **i32)
        self.used = torch.zeros(1, **i32)
        # the merge's two parts are fp32 tensors; the workspace splits long contexts
        self.ctx = hb.Context(torch.device(device).index, hb.hg_workspace_bytes(most_tokens, self.Hq, dim, 4))

    def prefill_system_prompt(self, Q):
        """Causal attention of the system prompt's own tokens: Q [P, Hq, D] (rows may lie further apart)."""
        k, v = self.system
        O = torch.empty(Q.shape, dtype=torch.bfloat16, device=Q.device)
        off = torch.tensor([0, Q.shape[0]], dtype=torch.int32, device=Q.device)
        hb.hg_prompt_attn(self.ctx, Q, k, v, off, Q.shape[0], O)
        return O

    def step(self, qkv, counts, most):
        """qkv [T, Hq + 2 Hkv, D]: the projection of the new tokens, request after request; counts: int32 [B] on the device, T in sum, none above `most`."""
        T, dev = qkv.shape[0], qkv.device
        Q, K, V = qkv[:, :self.Hq], qkv[:, self.Hq:self.Hq + self.Hkv], qkv[:, self.Hq + self.Hkv:]
        q_off, slots = torch.empty(self.B + 1, dtype=torch.int32, device=dev), torch.empty(T, dtype=torch.int32, device=dev)
        hb.hg_page_slots(self.ctx, self.lengths, counts, self.free, self.page_size, self.kv.page_table, q_off, slots, self.grown, self.used)
        hb.hg_kv_write_paged(self.ctx, K, V, slots, self.kv)
        O = [torch.empty(T, self.Hq, self.D, dtype=torch.float32, device=dev) for _ in range(2)]
        L = [torch.empty(T, self.Hq, dtype=torch.float32, device=dev) for _ in range(2)]
        hb.hg_chunk_attn_paged(self.ctx, Q, q_off, self.kv, self.grown, most, self.row_capacity, O[0], L[0])
        hb.hg_prefix_attn(self.ctx, Q.contiguous(), *self.system, O[1], L[1])
        out = torch.empty(T, self.Hq, self.D, dtype=torch.bfloat16, device=dev)
        hb.hg_merge(self.ctx, O, L, out)
        # The one look at the device.  A step in which some token has no place is not taken: lengths and free pages stay, and what it has written lies behind the requests' rows
        # or in pages that are still free, so it may be made again, with other counts or with more pages.
        taken, unplaced = torch.cat([self.used, (self.lengths + counts - self.grown).sum(0, keepdim=True, dtype=torch.int32)]).tolist()
        if taken > self.free.numel():
            raise RuntimeError(f"{taken} pages are wanted, {self.free.numel()} are free: admit fewer requests, or take pages back first")
        if unplaced:
            raise RuntimeError(f"{unplaced} tokens lie past the {self.row_capacity} rows that a request may have")
        self.lengths, self.grown = self.grown, self.lengths
        self.free = self.free[taken:]
        return out


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--requests", type=int, default=64)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--system", type=int, default=2048)
    ap.add_argument("--heads", default="32/8")
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--codes", action="store_true")
    a = ap.parse_args(argv)
    heads = tuple(int(x) for x in a.heads.split("/"))
    g = torch.Generator(device="cuda:0").manual_seed(0)
    rows = lambda T, H: torch.randn(T, H, a.dim, generator=g, device="cuda:0").to(torch.bfloat16)  # noqa: E731
    system = rows(a.system, heads[0] + 2 * heads[1])
    k, v = system[:, heads[0]:heads[0] + heads[1]].contiguous(), system[:, heads[0] + heads[1]:].contiguous()
    server = Server(a.requests, heads, a.dim, k, v, pages=a.requests * 64, codes=a.codes, row_capacity=1024)
    server.prefill_system_prompt(system[:, :heads[0]])
    # prompts of 1 to 512 tokens, then every request decodes
    prompts = [1 + 511 * i // max(a.requests - 1, 1) for i in range(a.requests)]
    for step in range(a.steps):
        counts = prompts if step == 0 else [1] * a.requests
        qkv, n = rows(sum(counts), heads[0] + 2 * heads[1]), torch.tensor(counts, dtype=torch.int32, device="cuda:0")
        torch.cuda.synchronize()
        t = time.perf_counter()
        server.step(qkv, n, max(counts))
        torch.cuda.synchronize()
        if step in (0, 1, a.steps - 1):
            print(f"step {step}: {sum(counts)} new tokens, {1e6 * (time.perf_counter() - t):.0f} us, {server.free.numel()} pages free", flush=True)


if __name__ == "__main__":
    main()
