"""The example that admits prompts into a running batch (examples/prompts_to_decode.py): every step's result is full attention of each token over the system
prompt and its own request's tokens so far."""
import os
import sys

import numpy as np
import pytest
import torch

import ragged_plain as plain
from parity import check

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("heads,dim,codes", [((8, 2), 128, False), ((16, 2), 64, False), ((4, 4), 128, True), ((8, 2), 64, True)])
def test_steps_of_a_running_batch(heads, dim, codes):
    from prompts_to_decode import Server
    Hq, Hkv = heads
    g = torch.Generator().manual_seed(1)
    rows = lambda T, H: torch.randn(T, H, dim, generator=g).to(torch.bfloat16)  # noqa: E731
    P, B = 300, 5
    system = rows(P, Hq + 2 * Hkv)
    dev = system.to("cuda:0")
    server = Server(B, heads, dim, dev[:, Hq:Hq + Hkv].contiguous(), dev[:, Hq + Hkv:].contiguous(), pages=60, row_capacity=512, codes=codes)
    got = server.prefill_system_prompt(dev[:, :Hq])
    sk, sv = system[:, Hq:Hq + Hkv].double(), system[:, Hq + Hkv:].double()
    O, L = plain.attention(system[:, :Hq], [0, P], [sk], [sv], [P])
    check(got.cpu().double().numpy(), None, O.numpy(), L.numpy(), "system prompt", out_bf16=True)

    def stored(x):
        if not codes:
            return x.double()
        s = float(np.float32(0.0125))
        return (x.float() / np.float32(0.0125)).clamp(-448, 448).to(torch.float8_e4m3fn).double() * s

    keys, values = [sk[:0]] * B, [sv[:0]] * B
    for counts in ([40, 0, 130, 1, 17], [1, 33, 1, 1, 0], [1, 1, 70, 1, 1], [1, 1, 1, 1, 1]):
        qkv = rows(sum(counts), Hq + 2 * Hkv)
        got = server.step(qkv.to("cuda:0"), torch.tensor(counts, dtype=torch.int32, device="cuda:0"), max(counts))
        off = np.concatenate([[0], np.cumsum(counts)])
        new = [qkv[a:z] for a, z in zip(off, off[1:])]
        keys = [torch.cat([k, stored(x[:, Hq:Hq + Hkv])]) for k, x in zip(keys, new)]
        values = [torch.cat([v, stored(x[:, Hq + Hkv:])]) for v, x in zip(values, new)]
        O, L = plain.attention(qkv[:, :Hq], off, [torch.cat([sk, k]) for k in keys], [torch.cat([sv, v]) for v in values], [P + k.shape[0] for k in keys])
        check(got.cpu().double().numpy(), None, O.numpy(), L.numpy(), f"step {counts}", out_bf16=True)
    assert server.lengths.tolist() == [43, 35, 202, 4, 19]


def test_a_pool_without_room_is_reported():
    from prompts_to_decode import Server
    k = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda:0")
    server = Server(2, (4, 2), 64, k, k, pages=3, row_capacity=64)
    qkv = torch.zeros(60, 8, 64, dtype=torch.bfloat16, device="cuda:0")
    with pytest.raises(RuntimeError, match="4 pages are wanted, 3 are free"):
        server.step(qkv, torch.tensor([30, 30], dtype=torch.int32, device="cuda:0"), 30)


def test_the_command_runs(capsys):
    import prompts_to_decode
    prompts_to_decode.main(["--requests", "6", "--steps", "3", "--system", "100"])
    assert "step 2: 6 new tokens" in capsys.readouterr().out
