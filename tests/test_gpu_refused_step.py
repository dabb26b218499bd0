"""A step that examples/prompts_to_decode.py refuses, because some token has no place, leaves the server as it was: the next ones are right."""
import os
import sys

import numpy as np
import pytest
import torch

import ragged_plain as plain
from parity import check

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("pages,capacity,refused,message", [(4, 128, [30, 50], "pages are wanted, 2 are free"), (4, 128, [0, 44], "3 pages are wanted, 2 are free"),
                                                            (9, 32, [20, 28], "1 tokens lie past the 32 rows")])
def test_a_refused_step_changes_nothing(pages, capacity, refused, message, codes):
    from prompts_to_decode import Server
    B, Hq, Hkv, D, P = 2, 4, 2, 64, 20
    g = torch.Generator().manual_seed(7)
    rows = lambda T: torch.randn(T, Hq + 2 * Hkv, D, generator=g).to(torch.bfloat16)  # noqa: E731
    system = rows(P)
    dev = system.to("cuda:0")
    server = Server(B, (Hq, Hkv), D, dev[:, Hq:Hq + Hkv].contiguous(), dev[:, Hq + Hkv:].contiguous(), pages=pages, row_capacity=capacity, codes=codes)
    sk, sv = system[:, Hq:Hq + Hkv].double(), system[:, Hq + Hkv:].double()

    def stored(x):
        return (x.float() / np.float32(0.0125)).clamp(-448, 448).to(torch.float8_e4m3fn).double() * float(np.float32(0.0125)) if codes else x.double()

    def step(counts, qkv):
        return server.step(qkv.to("cuda:0"), torch.tensor(counts, dtype=torch.int32, device="cuda:0"), max(counts))

    keys, values, lengths = [sk] * B, [sv] * B, [0] * B
    for counts in ([10, 5], refused, [6, 12], [1, 1] if pages > 4 else [0, 1]):
        qkv = rows(sum(counts))
        if counts is refused:
            free = server.free.clone()
            for _ in range(2):
                with pytest.raises(RuntimeError, match=message):
                    step(counts, qkv)
            assert server.lengths.tolist() == lengths and torch.equal(server.free, free)
            continue
        got = step(counts, qkv)
        off = np.concatenate([[0], np.cumsum(counts)])
        new = [qkv[a:z] for a, z in zip(off, off[1:])]
        keys = [torch.cat([k, stored(x[:, Hq:Hq + Hkv])]) for k, x in zip(keys, new)]
        values = [torch.cat([v, stored(x[:, Hq + Hkv:])]) for v, x in zip(values, new)]
        lengths = [n + c for n, c in zip(lengths, counts)]
        O, L = plain.attention(qkv[:, :Hq], off, keys, values, [P + n for n in lengths])
        check(got.cpu().double().numpy(), None, O.numpy(), L.numpy(), f"step {counts}", out_bf16=True)
        assert server.lengths.tolist() == lengths
        used = [p for row, n in zip(server.kv.page_table.tolist(), lengths) for p in row[:-(-n // 16)]]
        assert len(set(used)) == len(used) and not set(used) & set(server.free.tolist())
