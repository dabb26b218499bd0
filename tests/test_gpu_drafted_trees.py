"""The calls of a step over drafted trees as a server makes them (examples/drafted_trees.py): after several steps the caches hold the rows of what has been said and nothing else, and what has
been said is what the model says token by token."""
import os
import sys

import pytest
import torch

from paper_2402_05099_amd import binding as hb

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
DEV = "cuda:0"


def run(heads, dim, branches, codes, greedy, steps=9, B=5, layers=3, attends=1.0):
    from drafted_trees import Server, Toy
    model = Toy(layers, heads, dim, 60, 256, attends=attends)
    server = Server(model, B, branches, pages=B * 16, codes=codes, greedy=greedy)
    texts = [[0] for _ in range(B)]      # (the first token is 0, and has no row yet)
    for _ in range(steps):
        for text, new in zip(texts, server.step()):
            text.extend(new)
    return model, server, texts


def stored(x, codes):
    return (x.float() / torch.tensor(0.0125, device=DEV)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if codes else x


@pytest.mark.parametrize("greedy", [False, True])
@pytest.mark.parametrize("heads,dim,branches,codes", [((8, 2), 128, [3, 2, 2], False), ((4, 4), 64, [1, 1, 1, 1, 1], False), ((16, 2), 64, [4, 3], True), ((8, 1), 128, [2, 2, 2, 2, 2], True)])
def test_the_caches_hold_what_has_been_said(heads, dim, branches, codes, greedy):
    model, server, texts = run(heads, dim, branches, codes, greedy)
    assert [len(t) - 1 for t in texts] == server.lengths.tolist()      # the last token's row comes with the next step
    assert sum(len(t) for t in texts) > 1.2 * len(texts) * 9           # drafts have stood
    free = server.free.tolist()
    used = [p for b, n in enumerate(server.lengths.tolist()) for p in server.table[b, :-(-n // 16)].tolist()]
    assert sorted(free + used) == list(range(5 * 16))                  # every page has one owner
    for layer, kv in enumerate(server.kv):
        for b, text in enumerate(texts):
            n = len(text) - 1
            j = torch.arange(n, device=DEV)
            at = server.table[b, j // 16].long() * 16 + j % 16
            _, K, V = model.qkv(layer, torch.tensor(text[:n], device=DEV), j)
            assert torch.equal(kv.K[at], stored(K, codes)) and torch.equal(kv.V[at], stored(V, codes)), (layer, b)


@pytest.mark.parametrize("heads,dim,branches,codes", [((8, 2), 128, [3, 2, 2], False), ((16, 2), 64, [4, 3], True)])
def test_greedy_steps_say_what_single_tokens_say(heads, dim, branches, codes):
    """The scores of every token that was said, from the causal attention of the whole text: the one that was said is the best, but for the roundings of O, which are at most max(1e-2, 2^-7 |O|)
    an element on either side (the gates of parity.py; |O| <= 4 here) and meet the product's columns."""
    model, server, texts = run(heads, dim, branches, codes, True)
    kv, layer = server.kv[-1], model.layers - 1
    for b, text in enumerate(texts):
        n = len(text) - 1
        said, j = torch.tensor(text, device=DEV), torch.arange(n, device=DEV)
        Q = model.qkv(layer, said[:n], j)[0].contiguous()
        O = torch.empty(n, *Q.shape[1:], dtype=torch.float32, device=DEV)
        one = hb.PagedKV(K=kv.K, V=kv.V, page_table=kv.page_table[b:b + 1].contiguous(), page_size=16, kv_format=kv.kv_format, k_scale=kv.k_scale, v_scale=kv.v_scale)
        i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
        hb.hg_chunk_attn_paged(server.ctx, Q, i32(0, n), one, i32(n), n, n, O)
        scores = model.scores(said[:n], O)
        off = 2 * torch.clamp(O.abs().flatten(1) * 2 ** -7, min=1e-2) @ model.out.abs()
        got = scores.gather(1, said[1:, None])[:, 0]
        assert O.abs().max() <= 4
        assert torch.all(got + off.amax(1) * 2 >= scores.amax(1))


def test_a_step_without_pages_is_reported():
    from drafted_trees import Server, Toy
    server = Server(Toy(1, (4, 2), 64, 20, 64), 3, [2, 2], pages=2)
    with pytest.raises(RuntimeError, match="3 pages are wanted, 2 are free"):
        server.step()


def test_the_command_runs(capsys):
    import drafted_trees
    drafted_trees.main(["--requests", "4", "--steps", "3", "--layers", "2", "--vocabulary", "100"])
    drafted_trees.main(["--requests", "3", "--steps", "2", "--layers", "1", "--vocabulary", "100", "--greedy", "--codes", "--tree", "2,1"])
    assert capsys.readouterr().out.count("tokens a request and step") == 5
