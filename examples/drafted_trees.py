#!/usr/bin/env python3
"""Speculative decoding with trees: a drafting model proposes several continuations of every request, the target model looks at all of them in one pass, and what it would have said
itself stands.  The models are toys of random numbers (one is the other without its attention); the step is a server's:

  hg_page_slots        places for the trees' tokens behind the requests' rows
  hg_tree_masks        what each token follows from, and how far behind the context it would stand
  hg_kv_write_paged    their K and V rows to those places, layer by layer
  hg_tree_attn_paged   each token's attention over its request's rows and over those it follows from, layer by layer
  hg_tree_verify       which tokens stand, from the target's and the drafts' probabilities and random numbers, and the token behind them
  hg_tree_keep_paged   the rows of those that stand move together behind the context, in all layers at once

The host looks once a step, to take back the pages that the refused tokens had.

usage: drafted_trees.py [--requests N] [--steps K] [--layers L] [--tree 3,2,2] [--heads 32/8] [--dim 128] [--vocabulary V] [--codes] [--greedy]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2402_05099_amd import binding as hb  # noqa: E402


class Toy:
    """Random tables in the place of a model: Q, K and V of a token at a position, layer by layer, and the scores of what comes next, which the drafting model knows but for `attends` times a
    product with the last layer's attention."""

    def __init__(self, layers, heads, dim, vocabulary, positions, attends=1.0, sharp=3.0, seed=0, device="cuda:0"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.Hq, self.Hkv = heads
        table = lambda n: torch.randn(layers, n, heads[0] + 2 * heads[1], dim, generator=g, device=device).to(torch.bfloat16)  # noqa: E731
        self.token, self.position = table(vocabulary), table(positions)
        self.bigram = sharp * torch.randn(vocabulary, vocabulary, generator=g, device=device)
        self.out = attends * torch.randn(heads[0] * dim, vocabulary, generator=g, device=device) / (heads[0] * dim) ** 0.5
        self.layers, self.dim, self.vocabulary = layers, dim, vocabulary

    def qkv(self, layer, tokens, positions):
        x = (self.token[layer, tokens.long()] + self.position[layer, positions.long()]) * 0.7
        return x[:, :self.Hq], x[:, self.Hq:self.Hq + self.Hkv], x[:, self.Hq + self.Hkv:]

    def scores(self, tokens, O):
        return self.bigram[tokens.long()] + O.flatten(1).float() @ self.out

    def drafts(self, tokens):
        return torch.softmax(self.bigram[tokens.long()], 1)


def tree_of(branches):
    """Parents of a tree in which every token of level i has branches[i] children: those of a token lie behind each other, level by level."""
    parents, level = [-1], [0]
    for k in branches:
        level_of_children = []
        for p in level:
            for _ in range(k):
                level_of_children.append(len(parents))
                parents.append(p)
        level = level_of_children
    return parents


class Server:
    def __init__(self, model, requests, branches, pages, page_size=16, row_capacity=1024, codes=False, greedy=False, seed=0, device="cuda:0"):
        self.model, self.B, self.page_size, self.greedy = model, requests, page_size, greedy
        self.row_capacity = row_capacity
        i32 = dict(dtype=torch.int32, device=device)
        self.tree = tree_of(branches)
        n = self.n = len(self.tree)
        T = requests * n
        self.parents = torch.tensor(self.tree * requests, **i32)
        self.children = [torch.tensor([t for t in range(n) if self.tree[t] == p], dtype=torch.long, device=device) for p in range(n)]
        self.first = torch.arange(requests, device=device) * n
        self.g = torch.Generator(device=device).manual_seed(seed)
        dtype = torch.uint8 if codes else torch.bfloat16
        table = torch.full((requests, row_capacity // page_size), -1, **i32)
        self.kv = [hb.PagedKV(K=torch.zeros(pages * page_size, model.Hkv, model.dim, dtype=dtype, device=device), V=torch.zeros(pages * page_size, model.Hkv, model.dim, dtype=dtype, device=device),
                              page_table=table, page_size=page_size, kv_format=hb.HG_KV_E4M3 if codes else hb.HG_KV_BF16, k_scale=0.0125, v_scale=0.0125) for _ in range(model.layers)]
        self.table, self.free = table, torch.arange(pages, **i32)
        self.lengths, self.grown, self.kept_lengths = (torch.zeros(requests, **i32) for _ in range(3))
        self.counts, self.used = torch.full((requests,), n, **i32), torch.zeros(1, **i32)
        self.q_off, self.slots = torch.empty(requests + 1, **i32), torch.empty(T, **i32)
        self.masks, self.depth = torch.empty(T, -(-n // 32), **i32), torch.empty(T, **i32)
        self.path, self.accepted, self.next = torch.empty(T, **i32), torch.empty(requests, **i32), torch.zeros(requests, **i32)
        self.ctx = hb.Context(torch.device(device).index, hb.hg_workspace_bytes(T, model.Hq, model.dim, 8))

    def draft(self):
        """Tokens of the trees, [B * n], and the probabilities that each token's children were drawn with"""
        tokens = torch.zeros(self.B, self.n, dtype=torch.int64, device=self.parents.device)
        tokens[:, 0] = self.next
        probabilities = torch.empty(self.B, self.n, self.model.vocabulary, device=tokens.device)
        for p in range(self.n):
            probabilities[:, p] = self.model.drafts(tokens[:, p])
            if len(self.children[p]):
                many = len(self.children[p])
                tokens[:, self.children[p]] = (torch.topk(probabilities[:, p], many).indices if self.greedy else
                                               torch.multinomial(probabilities[:, p], many, replacement=True, generator=self.g))
        return tokens.to(torch.int32).view(-1), probabilities.view(self.B * self.n, -1)

    def step(self):
        """One step of all requests: the lists of tokens that each has said."""
        m, ctx, T = self.model, self.ctx, self.B * self.n
        tokens, drafts = self.draft()
        hb.hg_page_slots(ctx, self.lengths, self.counts, self.free, self.page_size, self.table, self.q_off, self.slots, self.grown, self.used)
        hb.hg_tree_masks(ctx, self.parents, self.q_off, self.n, self.masks, self.depth)
        positions = self.lengths.repeat_interleave(self.n) + self.depth
        O = torch.empty(T, m.Hq, m.dim, dtype=torch.bfloat16, device=tokens.device)
        for layer, kv in enumerate(self.kv):
            Q, K, V = m.qkv(layer, tokens, positions)
            hb.hg_kv_write_paged(ctx, K, V, self.slots, kv)
            hb.hg_tree_attn_paged(ctx, Q, self.q_off, self.masks, kv, self.grown, self.n, self.row_capacity, O)
        scores = m.scores(tokens, O)
        if self.greedy:
            hb.hg_tree_verify(ctx, tokens, self.parents, self.q_off, self.n, scores.argmax(1).to(torch.int32), None, None, None, self.path, self.accepted, self.next)
        else:
            u, u_next = torch.rand(T, generator=self.g, device=tokens.device), torch.rand(self.B, generator=self.g, device=tokens.device)
            hb.hg_tree_verify(ctx, tokens, self.parents, self.q_off, self.n, torch.softmax(scores, 1), drafts, u, u_next, self.path, self.accepted, self.next)
        hb.hg_tree_keep_paged(ctx, self.kv, self.q_off, self.path, self.accepted, self.grown, self.n, self.kept_lengths)
        # the one look at the device
        taken, unplaced = torch.cat([self.used, (self.lengths + self.counts - self.grown).sum(0, keepdim=True, dtype=torch.int32)]).tolist()
        if taken > self.free.numel():
            raise RuntimeError(f"{taken} pages are wanted, {self.free.numel()} are free")
        if unplaced:
            raise RuntimeError(f"{unplaced} tokens lie past the {self.row_capacity} rows that a request may have")
        # pages behind the kept rows are free again
        entry, ps = torch.arange(self.table.shape[1], device=tokens.device), self.page_size
        behind = (entry >= ((self.kept_lengths + ps - 1) // ps)[:, None]) & (entry < ((self.grown + ps - 1) // ps)[:, None])
        self.free = torch.cat([self.free[taken:], self.table[behind]])
        self.lengths, self.kept_lengths = self.kept_lengths, self.lengths
        path, said = self.path.view(self.B, self.n).tolist(), tokens.view(self.B, self.n).tolist()
        return [[said[b][t] for t in path[b][1:] if t >= 0] + [nxt] for b, nxt in enumerate(self.next.tolist())]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--requests", type=int, default=32)
    ap.add_argument("--steps", type=int, default=24)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--tree", default="3,2,2")
    ap.add_argument("--heads", default="32/8")
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--vocabulary", type=int, default=2000)
    ap.add_argument("--codes", action="store_true")
    ap.add_argument("--greedy", action="store_true")
    a = ap.parse_args(argv)
    model = Toy(a.layers, tuple(int(x) for x in a.heads.split("/")), a.dim, a.vocabulary, 4096)
    server = Server(model, a.requests, [int(k) for k in a.tree.split(",")], pages=a.requests * 40, codes=a.codes, greedy=a.greedy)
    said = 0
    for step in range(a.steps):
        torch.cuda.synchronize()
        t = time.perf_counter()
        said += sum(len(x) for x in server.step())
        us = 1e6 * (time.perf_counter() - t)
        if step in (0, 1, a.steps - 1):
            print(f"step {step}: {us:.0f} us, {said / (step + 1) / a.requests:.2f} tokens a request and step", flush=True)


if __name__ == "__main__":
    main()
