"""CPU: what the operators of a speculative step refuse, at the C ABI (before any device work) and in
the binding."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2603_23049_amd import pcr

INV, UNS, OK = pcr.PCR_ERR_INVALID_ARG, pcr.PCR_ERR_UNSUPPORTED, pcr.PCR_OK
A = 0x10000          # an aligned address that is never read


def _tree(**kw):
    a = dict(B=2, cu=A, par=A, p=A, T=10, words=1, vis=A, pos=A)
    a.update(kw)
    return pcr.lib().pcr_draft_tree(*a.values(), None)


@pytest.mark.parametrize("kw,st", [(dict(B=-1), INV), (dict(T=-1), INV), (dict(words=0), UNS), (dict(words=17), UNS),
                                   (dict(B=2 ** 21 + 1), UNS), (dict(T=2 ** 27 + 1), UNS), (dict(cu=None), INV),
                                   (dict(par=None), INV), (dict(p=None), INV), (dict(vis=None), INV),
                                   (dict(pos=None), INV), (dict(vis=A + 4), INV), (dict(B=0), OK), (dict(T=0), OK)])
def test_draft_tree(kw, st):
    assert _tree(**kw) == st and (st == OK or pcr.last_error())


def _pool(nb=4, Hkv=2, d=64, bs=16, k=A, v=A << 8):
    return pcr._Pool(k, v, nb, bs, Hkv, d)


def _attn(pool=None, **kw):
    pl, cu = np.array(kw.pop("pl", [20, 0]), np.int32), np.array(kw.pop("n_cu", [0, 5, 9]), np.int32)
    a = dict(q=A, bt=A, mb=4, p=A, cu=A, hpl=pl.ctypes.data, hcu=cu.ctypes.data, B=2, vis=A, words=1, Hq=4, scale=0.1,
             out=A << 4, ws=A, wsb=1 << 40)
    a.update(kw)
    pool = pool or _pool()
    v = list(a.values())
    return pcr.lib().pcr_tree_attn(v[0], ctypes.byref(pool), *v[1:], None)


@pytest.mark.parametrize("kw,st", [
    (dict(B=-1), INV), (dict(hpl=None), INV), (dict(hcu=None), INV), (dict(Hq=3), UNS), (dict(Hq=0), UNS),
    (dict(scale=0.0), INV), (dict(scale=float("nan")), INV), (dict(scale=float("inf")), INV), (dict(words=0), UNS),
    (dict(words=17), UNS), (dict(n_cu=[1, 5, 9]), INV), (dict(n_cu=[0, 5, 4]), INV), (dict(pl=[-1, 0]), INV),
    (dict(pl=[60, 0]), INV), (dict(n_cu=[0, 65, 65], mb=9), INV), (dict(pl=[2 ** 30, 0], mb=2 ** 27), UNS),
    (dict(pl=[2 ** 31 - 1, 0], mb=2 ** 27), UNS),
    (dict(q=None), INV), (dict(out=None), INV), (dict(bt=None), INV), (dict(p=None), INV), (dict(cu=None), INV),
    (dict(vis=None), INV), (dict(q=A + 8), INV), (dict(out=A + 2), INV), (dict(vis=A + 4), INV), (dict(out=A), INV),
    (dict(out=A + 1024), INV), (dict(B=0), OK), (dict(n_cu=[0, 0, 0]), OK)])
def test_tree_attn(kw, st):
    assert _attn(**kw) == st and (st == OK or pcr.last_error())


def test_tree_attn_pools():
    for pool, st in ((_pool(k=None), INV), (_pool(nb=0), INV), (_pool(d=96), UNS), (_pool(bs=8), UNS), (_pool(v=A + 4), INV)):
        assert _attn(pool) == st


def test_workspace_sizes():
    n = ctypes.c_int64(0)
    f = pcr.lib().pcr_tree_attn_workspace_size
    assert f(1, 1, 4, 2, 64, 10, None) == INV and f(-1, 1, 4, 2, 64, 10, ctypes.byref(n)) == INV
    assert f(1, -1, 4, 2, 64, 10, ctypes.byref(n)) == INV and f(1, 1, 4, 2, 64, -1, ctypes.byref(n)) == INV
    assert f(1, 1, 5, 2, 64, 10, ctypes.byref(n)) == UNS and f(1, 1, 4, 2, 80, 10, ctypes.byref(n)) == UNS
    for empty in ((0, 9, 4, 2, 64, 9), (2, 0, 4, 2, 64, 9), (2, 9, 4, 2, 64, 0)):
        assert f(*empty, ctypes.byref(n)) == OK and n.value == 0
    f = pcr.lib().pcr_verify_drafts_workspace_size
    assert f(1, 1, 10, None) == INV and f(-1, 1, 10, ctypes.byref(n)) == INV and f(1, 1, 0, ctypes.byref(n)) == INV
    assert f(1, -1, 10, ctypes.byref(n)) == INV
    assert f(0, 0, 10, ctypes.byref(n)) == OK and n.value == 0


def _verify(**kw):
    a = dict(B=2, cu=A, par=A, tok=A, T=10, V=100, tp=A, ts=100, dp=A, ds=100, u=A, p=A, cap=4, path=A, acc=A, nxt=A, ctx=A,
             ws=A, wsb=1 << 40)
    a.update(kw)
    return pcr.lib().pcr_verify_drafts(*a.values(), None)


@pytest.mark.parametrize("kw,st", [
    (dict(B=-1), INV), (dict(T=-1), INV), (dict(V=0), INV), (dict(cap=0), INV), (dict(ts=99), INV), (dict(ds=99), INV),
    (dict(ts=2 ** 32 + 1), UNS), (dict(ds=2 ** 32 + 1), UNS), (dict(V=2 ** 30 + 1, ts=2 ** 31, ds=2 ** 31), UNS),
    (dict(B=2 ** 21 + 1), UNS), (dict(T=2 ** 27 + 1), UNS), (dict(cu=None), INV), (dict(par=None), INV),
    (dict(tok=None), INV), (dict(tp=None), INV), (dict(u=None), INV), (dict(p=None), INV), (dict(path=None), INV),
    (dict(acc=None), INV), (dict(nxt=None), INV), (dict(ctx=None), INV), (dict(B=0), OK)])
def test_verify_drafts(kw, st):
    assert _verify(**kw) == st and (st == OK or pcr.last_error())


def _compact(of=None, **kw):
    of = [_pool(), _pool(k=A << 12, v=A << 14)] if of is None else of
    arr = (pcr._Pool * max(1, len(of)))(*of)
    a = dict(pools=ctypes.addressof(arr), L=len(of), bt=A, mb=4, p=A, path=A, cap=3, acc=A, B=2)
    a.update(kw)
    return pcr.lib().pcr_compact_kv(*a.values(), None)


@pytest.mark.parametrize("kw,st", [(dict(pools=None), INV), (dict(L=-1), INV), (dict(L=257), UNS), (dict(bt=None), INV),
                                   (dict(mb=0), INV), (dict(p=None), INV), (dict(path=None), INV), (dict(cap=0), INV),
                                   (dict(acc=None), INV), (dict(B=-1), INV), (dict(B=65536), UNS), (dict(B=0), OK),
                                   (dict(L=0), OK)])
def test_compact_kv(kw, st):
    assert _compact(**kw) == st and (st == OK or pcr.last_error())


def test_compact_kv_pools():
    far = _pool(k=A << 12, v=A << 14)
    for other in (_pool(nb=5, k=far.k, v=far.v), _pool(Hkv=1, k=far.k, v=far.v), _pool(d=128, k=far.k, v=far.v),
                  _pool(v=far.v), _pool(k=far.k), _pool(k=A + 4 * 2 * 16 * 64 * 2 - 16, v=far.v), _pool(k=far.k, v=far.k),
                  _pool(k=None, v=far.v)):
        assert _compact([_pool(), other]) == INV and pcr.last_error()
    assert _compact([_pool(nb=2 ** 27 + 1, Hkv=1, k=A << 24, v=A << 36)]) == UNS
    assert _compact([_pool(), _pool(d=80, k=far.k, v=far.v)]) == UNS


def _bt(B=2, w=4):
    return torch.zeros(B, w, dtype=torch.int32)


def test_binding():
    """Arrays of the wrong type, order, length or place (here every tensor is on the CPU)."""
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)         # noqa: E731
    w = torch.zeros(10, 1, dtype=torch.int64)
    for vis in (torch.zeros(10, 1, dtype=torch.int32), torch.zeros(9, 1, dtype=torch.int64), torch.zeros(10, dtype=torch.int64), w):
        with pytest.raises(ValueError, match="visible"):
            pcr.draft_tree(i(3), i(10), i(2), vis, i(10))
    pool = pcr.KVPool(torch.zeros(4, 2, 1024, dtype=torch.bfloat16), torch.zeros(4, 2, 1024, dtype=torch.bfloat16), 2, 64)
    q = torch.zeros(9, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="host_cu_nodes"):
        pcr.tree_attn(q, pool, _bt(), i(2), i(3), [20, 0], [0, 5], w, 4, q.clone())
    with pytest.raises(ValueError, match="block_tables"):
        pcr.tree_attn(q, pool, i(8), i(2), i(3), [20, 0], [0, 5, 9], w, 4, q.clone())
    with pytest.raises(ValueError, match="current GPU"):
        pcr.tree_attn(q, pool, _bt(), i(2), i(3), [20, 0], [0, 5, 9], w, 4, q.clone())
    with pytest.raises(ValueError, match="q holds"):
        pcr.tree_attn(q.half(), pool, _bt(), i(2), i(3), [20, 0], [0, 5, 9], w, 4, q.clone())
    f = torch.zeros(10, 50)
    ok = dict(cu_nodes=i(3), parents=i(10), tokens=i(10), target_probs=f, draft_probs=None, uniforms=torch.zeros(10),
              prefix_lens=i(2), path=i(2, 4), accepted_lens=i(2), next_tokens=i(2), context_lens=i(2))
    for kw, what in ((dict(target_probs=f.double()), "target_probs"), (dict(target_probs=f[:9]), "target_probs"),
                     (dict(target_probs=torch.zeros(50, 10).t()), "target_probs"), (dict(target_probs=f[0]), "target_probs"),
                     (dict(path=i(8)), "path"), (dict(), "current GPU")):
        with pytest.raises(ValueError, match=what):
            pcr.verify_drafts(**{**ok, **kw})
    with pytest.raises(ValueError, match="pool.k"):
        pcr.KVLayers([pool])
    layers = pcr.KVLayers([])
    with pytest.raises(ValueError, match="path"):
        pcr.compact_kv(layers, _bt(), i(2), i(8), i(2))
