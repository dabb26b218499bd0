"""What the calls of a decode step over drafted trees refuse, and what they accept without doing anything.  No kernel is launched here: the checks come before any device work, so the
context may be an empty one."""
import ctypes

import pytest
import torch

from paper_2402_05099_amd import binding as hb

OK, BAD, NOT = hb.HG_OK, hb.HG_ERR_INVALID_ARG, hb.HG_ERR_UNSUPPORTED
CTX = (ctypes.c_char * 4096)()      # an empty context: nothing of it is looked at before the checks have passed
ctx = ctypes.addressof(CTX)
A, B_, C, D_, E, F, G_, H_, I_, J_ = (0x10000 * (i + 1) for i in range(10))      # addresses that nothing reads


def masks(c=ctx, parents=A, q_off=B_, rows=8, max_new=8, B=2, out=C, words=1, depth=D_):
    return hb.lib().hg_tree_masks(c, parents, q_off, rows, max_new, B, out, words, depth)


def test_masks():
    for bad in (dict(c=None), dict(rows=-1), dict(max_new=-1), dict(B=-1), dict(q_off=None), dict(parents=None), dict(out=None), dict(words=-1), dict(words=0), dict(rows=70, max_new=33),
                dict(out=A), dict(out=B_), dict(depth=C), dict(depth=A)):
        assert masks(**bad) == BAD, bad
    for bad in (dict(max_new=hb.HG_MAX_TREE + 1), dict(B=1 << 22), dict(words=1 << 21)):
        assert masks(**bad) == NOT, bad
    for nothing in (dict(rows=0, parents=None, out=None, words=0), dict(B=0, q_off=None), dict(max_new=0)):
        assert masks(**nothing) == OK, nothing


def paged(**more):
    f = dict(K=F, V=G_, page_table=H_, page_size=16, table_stride=4, n_pages=8, kv_format=hb.HG_KV_BF16, k_scale=1.0, v_scale=1.0)
    f.update(more)
    return hb.hg_paged_kv(*[f[n] for n, _ in hb.hg_paged_kv._fields_])


def attn(c=ctx, Q=A, step=8 * 128, q_off=B_, rows=8, m=C, words=1, lengths=D_, max_new=8, max_len=64, B=2, Hq=8, Hkv=2, D=128, O=E, dtype=hb.HG_BF16, kv=None, **cache):
    st = paged(**cache)
    return hb.lib().hg_tree_attn_paged(c, Q, step, q_off, rows, m, words, ctypes.byref(st) if kv is None else kv, lengths, max_new, max_len, B, Hq, Hkv, D, 0.0, O, dtype, None)


def test_attention():
    for bad in (dict(c=None), dict(m=None), dict(words=0), dict(words=-1), dict(rows=80, max_new=33), dict(Q=None), dict(Q=A + 2), dict(q_off=None), dict(lengths=None), dict(O=None), dict(O=E + 8),
                dict(step=8 * 128 - 8), dict(step=8 * 128 + 4), dict(rows=-1), dict(max_new=-1), dict(max_len=-1), dict(B=-1), dict(Hq=0), dict(Hkv=0), dict(dtype=2), dict(K=None), dict(V=G_ + 4),
                dict(page_table=None), dict(page_size=24), dict(page_size=8), dict(n_pages=0), dict(n_pages=-1), dict(table_stride=3), dict(kv_format=5), dict(kv_format=1, k_scale=0.0),
                dict(kv_format=1, v_scale=float("nan"))):
        assert attn(**bad) == BAD, bad
    for bad in (dict(D=96), dict(Hq=9), dict(words=1 << 26), dict(n_pages=1 << 27), dict(rows=1 << 29, words=1 << 20), dict(max_len=1 << 30, table_stride=1 << 26)):
        assert attn(**bad) == NOT, bad
    for nothing in (dict(rows=0, m=None, words=0), dict(B=0), dict(max_new=0)):
        assert attn(**nothing) == OK, nothing
    assert hb.lib().hg_tree_attn_paged(ctx, A, 1024, B_, 8, C, 1, None, D_, 8, 64, 2, 8, 2, 128, 0.0, E, 1, None) == BAD


def verify(c=ctx, tokens=A, parents=B_, q_off=C, rows=8, max_new=8, B=2, V=100, target=D_, t_step=100, draft=E, d_step=100, kind=hb.HG_F32, u=F, u_next=G_, path=H_, kept=I_, nxt=J_):
    return hb.lib().hg_tree_verify(c, tokens, parents, q_off, rows, max_new, B, V, target, t_step, draft, d_step, kind, u, u_next, path, kept, nxt)


def test_verification():
    names = ("tokens", "parents", "q_off", "target", "u", "u_next", "path", "kept", "nxt")
    for bad in [{n: None} for n in names] + [dict(c=None), dict(rows=-1), dict(max_new=-1), dict(B=-1), dict(V=0), dict(t_step=99), dict(d_step=99), dict(kind=3), dict(kind=-1), dict(target=D_ + 2),
                                             dict(draft=E + 1, kind=hb.HG_BF16), dict(path=A), dict(kept=C), dict(nxt=I_), dict(path=J_), dict(nxt=G_), dict(kept=D_)]:
        assert verify(**bad) == BAD, bad
    for bad in (dict(max_new=hb.HG_MAX_TREE + 1), dict(B=1 << 22), dict(V=1 << 30, t_step=1 << 30, d_step=1 << 30)):
        assert verify(**bad) == NOT, bad
    assert verify(B=0, q_off=None, kept=None) == OK
    greedy = dict(kind=hb.HG_TOKENS, V=0, t_step=0, draft=None, d_step=0, u=None, u_next=None)
    assert verify(**greedy, tokens=None) == BAD and verify(**greedy, path=D_) == BAD and verify(**greedy, B=0) == OK


def keep(c=ctx, layers=2, q_off=A, rows=8, path=B_, kept=C, lengths=D_, max_new=8, B=2, Hkv=2, D=128, grown=E, kvs=None, second=None, **cache):
    st = kvs or (hb.hg_paged_kv * 2)(paged(**cache), paged(**{**dict(K=I_, V=J_), **cache, **(second or {})}))
    return hb.lib().hg_tree_keep_paged(c, layers, st, q_off, rows, path, kept, lengths, max_new, B, Hkv, D, grown)


def test_the_move():
    for bad in [{n: None} for n in ("c", "q_off", "path", "kept", "lengths", "grown")] + [
            dict(layers=-1), dict(rows=-1), dict(max_new=-1), dict(B=-1), dict(Hkv=0), dict(grown=A), dict(grown=B_), dict(grown=C), dict(grown=D_), dict(grown=H_), dict(K=None), dict(K=I_ + 8),
            dict(page_size=24), dict(kv_format=2), dict(n_pages=-1), dict(table_stride=-1), dict(page_table=None),
            dict(second=dict(K=F)), dict(second=dict(V=F)), dict(K=F, V=F), dict(second=dict(page_table=I_)), dict(second=dict(page_size=32)), dict(second=dict(n_pages=7)),
            dict(second=dict(table_stride=5)), dict(second=dict(kv_format=1))]:
        assert keep(**bad) == BAD, bad
    for bad in (dict(layers=hb.HG_MAX_LAYERS + 1), dict(D=96), dict(max_new=hb.HG_MAX_TREE + 1), dict(B=1 << 22), dict(n_pages=1 << 27), dict(Hkv=1 << 17), dict(B=(1 << 22) - 1, Hkv=64)):
        assert keep(**bad) == NOT, bad
    assert keep(B=0, q_off=None, kept=None) == OK
    assert hb.lib().hg_tree_keep_paged(ctx, 1, None, A, 8, B_, C, D_, 8, 2, 2, 128, E) == BAD


def test_what_the_binding_refuses():
    n, kv = torch.zeros(2, dtype=torch.int32), hb.PagedKV(torch.zeros(16, 2, 64, dtype=torch.bfloat16), torch.zeros(16, 2, 64, dtype=torch.bfloat16), torch.zeros(1, 1, dtype=torch.int32), 16)
    q, p = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 5)
    for call in (lambda: hb.hg_tree_masks(None, n, n, 2, n.view(2, 1)), lambda: hb.hg_tree_attn_paged(None, q, n, n.view(2, 1), kv, n[:1], 2, 16, q),
                 lambda: hb.hg_tree_verify(None, n, n, n, 2, p, None, p[:, 0], p[:1, 0], n, n[:1], n[:1]), lambda: hb.hg_tree_keep_paged(None, [kv], n, n, n[:1], n[:1], 2, n[:1])):
        with pytest.raises((TypeError, ValueError), match="device tensor"):
            call()
    m = hb.native()
    assert m.tree_masks(None, n, n, 2, n, n) is None and m.tree_attn() is None and m.tree_verify(*[object()] * 12) is None and m.tree_keep(None, [], n, n, n, n, 2, n) is None
