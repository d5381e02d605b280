"""CPU: what the operators around the pool refuse, at the C ABI (before any device work) and in
the binding (arrays of the wrong type, order, length or place)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2603_23049_amd import pcr

INV, UNS = pcr.PCR_ERR_INVALID_ARG, pcr.PCR_ERR_UNSUPPORTED
A = 0x10000          # an aligned address that is never read


def _pool(nb=4, Hkv=2, d=64, bs=16):
    return ctypes.byref(pcr._Pool(A, A << 4, nb, bs, Hkv, d))


def _assign(**kw):
    a = dict(B=2, p=A, s=A, bt=A, mb=4, bs=16, nb=8, free=A, cap=8, cnt=A, slots=A, pos=None, scap=4, cu=A, ctx=A,
             out=A, status=A)
    a.update(kw)
    return pcr.lib().pcr_assign_blocks(*a.values(), None)


def _release(**kw):
    a = dict(B=2, n=A, keep=A, bt=A, mb=4, bs=16, nb=8, free=A, cap=8, cnt=A, out=A, status=A)
    a.update(kw)
    return pcr.lib().pcr_release_blocks(*a.values(), None)


@pytest.mark.parametrize("call", [_assign, _release])
@pytest.mark.parametrize("kw,st", [(dict(B=-1), INV), (dict(B=2 ** 30 + 1), UNS), (dict(mb=2 ** 27), UNS), (dict(cap=2 ** 30 + 1), UNS),
                                   (dict(mb=0), INV), (dict(nb=0), INV), (dict(bs=0), INV),
                                   (dict(bs=32), UNS), (dict(nb=2 ** 27 + 1), UNS), (dict(cap=-1), INV),
                                   (dict(bt=None), INV), (dict(free=None), INV), (dict(cnt=None), INV),
                                   (dict(out=None), INV), (dict(status=None), INV)])
def test_tables(call, kw, st):
    assert call(**kw) == st and pcr.last_error()


def test_assign_only():
    for kw in (dict(scap=-1), dict(p=None), dict(s=None), dict(slots=None), dict(cu=None), dict(ctx=None)):
        assert _assign(**kw) == INV
    assert _assign(scap=2 ** 30 + 1) == UNS and _assign(B=0, scap=0) == pcr.PCR_OK
    for kw in (dict(n=None), dict(keep=None)):
        assert _release(**kw) == INV


def _rope(rd=64, axes=1, axis=None, f=None, scale=1.0, inter=0):
    f = np.ones(max(rd // 2, 1), np.float32) if f is None else f
    r = pcr._Rope(f.ctypes.data, None if axis is None else axis.ctypes.data, rd, axes, inter, scale)
    r.keep = (f, axis)
    return r


def _append(rope=None, pool=None, **kw):
    a = dict(q=A, qs=256, k=A << 1, ks=128, v=A << 1, vs=128, pos=A, ps=10, slots=A, T=10, Hq=4, out=A << 8)
    a.update(kw)
    rope = _rope() if rope is None else rope
    return pcr.lib().pcr_rope_append_kv(ctypes.addressof(rope), pool or _pool(), *a.values(), None)


def _rows(rope=None, **kw):
    a = dict(x=A, xs=128, pos=A, ps=10, T=10, H=2, d=64, inv=0, out=A << 8, os=128)
    a.update(kw)
    rope = _rope() if rope is None else rope
    return pcr.lib().pcr_rope_rows(ctypes.addressof(rope), *a.values(), None)


@pytest.mark.parametrize("call", [_append, _rows])
def test_rotation(call):
    bad = np.ones(32, np.float32)
    bad[7] = np.inf
    nan = np.full(32, np.nan, np.float32)
    axis = np.zeros(32, np.int32)
    axis[3] = 2
    for r, st in ((_rope(rd=0), UNS), (_rope(rd=24), UNS), (_rope(rd=80), UNS), (_rope(rd=-16), UNS),
                  (_rope(axes=0), INV), (_rope(axes=5), INV), (_rope(scale=float("nan")), INV), (_rope(f=bad), INV),
                  (_rope(f=nan), INV), (_rope(axes=2, axis=axis), INV), (_rope(axis=-axis), INV)):
        assert call(rope=r) == st
    null = pcr._Rope(None, None, 64, 1, 0, 1.0)
    assert call(rope=null) == INV
    assert call(T=-1) == INV and call(T=0) == pcr.PCR_OK
    assert call(rope=_rope(axes=2), ps=9) == INV
    assert call(pos=None) == INV


def test_append_rows():
    for kw in (dict(qs=255), dict(qs=248), dict(ks=120), dict(vs=132), dict(q=A + 8), dict(k=A + 2), dict(v=None),
               dict(out=A + 4), dict(out=A), dict(out=A + 512), dict(slots=None), dict(q=None), dict(Hq=-4),
               dict(ks=(1 << 40) + 8)):
        if kw == dict(out=A):
            kw = dict(out=A, qs=264)                 # the same array, but not back to back
        assert _append(**kw) == INV, kw
    inside = A + 8192                                # of the pool's K: 4 blocks of 4 KB
    for kw in (dict(out=A + 16368), dict(k=inside), dict(v=inside), dict(v=(A << 4) + 16368), dict(out=(A << 4) - 16),
               dict(out=(A << 1) - 16), dict(k=(A << 8) + 16, ks=1024), dict(v=(A << 8) + 5104)):
        assert _append(**kw, q=A << 12) == INV and "overlap" in pcr.last_error(), kw
    assert _append(Hq=3) == UNS and _append(T=2 ** 27 + 1, ps=2 ** 28) == UNS
    assert _append(pool=_pool(d=96)) == UNS and _append(pool=_pool(bs=8)) == UNS
    assert pcr.lib().pcr_rope_append_kv(None, _pool(), A, 256, A, 128, A, 128, A, 10, A, 10, 4, A << 8, None) == INV


def test_plain_rows():
    for kw in (dict(H=0), dict(x=None), dict(out=None), dict(xs=120), dict(os=127), dict(x=A + 2), dict(out=A + 256),
               dict(out=A, os=136)):
        assert _rows(**kw) == INV, kw
    # parts of the same rows: overlapping by 8 elements at either end, or whole rows apart
    for kw in (dict(xs=256, os=256, out=A + 240), dict(xs=256, os=256, x=A + 272, out=A), dict(out=A + 512 * 3, xs=256, os=256),
               dict(out=A + 512 * 3 + 272, xs=256, os=256)):
        assert _rows(**kw) == INV and "overlap" in pcr.last_error(), kw
    assert _rows(T=2 ** 27 + 1, ps=2 ** 28) == UNS and _rows(H=2 ** 25, xs=2 ** 31, os=2 ** 31) == UNS
    for d in (0, 8, 72, 272, -16):
        assert _rows(d=d) == UNS
    assert _rows(rope=_rope(rd=64), d=48) == UNS


def _cross(n=(5, 9), cu=(0, 1, 3), **kw):
    n, cu = np.array(n, np.int32), np.array(cu, np.int32)
    a = dict(q=A, pool=_pool(), bt=A, mb=4, n=A, cu=A, hn=n.ctypes.data, hcu=cu.ctypes.data, B=len(n), Hq=4,
             scale=0.125, out=A << 8, ws=None, wsb=0)
    a.update(kw)
    return pcr.lib().pcr_cross_attn(*a.values(), None)


def test_cross():
    for kw in (dict(B=-1), dict(hn=None), dict(hcu=None), dict(scale=0.0), dict(scale=float("nan")), dict(scale=1e31),
               dict(cu=(1, 2, 3)), dict(cu=(0, 3, 1)), dict(n=(5, -1)), dict(n=(65, 9)), dict(q=None), dict(out=None),
               dict(bt=None), dict(cu=(0, 1, 2 ** 31 - 1)), dict(q=A + 2), dict(out=A + 4), dict(out=A + 512),
               dict(pool=None)):
        assert _cross(**kw) == INV, kw
    for kw in (dict(Hq=3), dict(Hq=0), dict(pool=_pool(d=80)), dict(pool=_pool(bs=32)), dict(n=(5, 2 ** 30 + 1), mb=2 ** 27),
               dict(B=2 ** 22, pool=_pool(Hkv=2))):
        assert _cross(**kw) == UNS, kw
    assert _cross(B=0) == pcr.PCR_OK and _cross(cu=(0, 0, 0)) == pcr.PCR_OK


def test_cross_workspace_size():
    n = ctypes.c_int64(-1)
    f = pcr.lib().pcr_cross_attn_workspace_size
    assert f(1, 1, 8, 2, 64, 100, None) == INV
    for a in ((-1, 1, 8, 2, 64, 10), (1, -1, 8, 2, 64, 10), (1, 1, 8, 2, 64, -1)):
        assert f(*a, ctypes.byref(n)) == INV
    for a in ((1, 1, 7, 2, 64, 10), (1, 1, 8, 2, 96, 10), (1, 1, 0, 2, 64, 10)):
        assert f(*a, ctypes.byref(n)) == UNS
    assert f(0, 0, 8, 2, 64, 0, ctypes.byref(n)) == pcr.PCR_OK and n.value == 0


# ---- the binding: CPU tensors (never reaching the library) ----

def _i(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_binding_tables():
    cpu = (torch, -1)                                    # as if CPU tensors were on the current GPU
    pcr._ints(cpu, 3, _i(3), "x")
    for x, msg in ((_i(2), "x holds 2 elements, the call takes 3"), (torch.zeros(3, dtype=torch.int64), "int64"),
                   (torch.zeros(3), "float32"), (_i(6)[::2], "not contiguous")):
        with pytest.raises(ValueError, match=msg):
            pcr._ints(cpu, 3, x, "x")
    with pytest.raises(ValueError, match="prefix_lens is on cpu, not on the current GPU"):
        pcr.assign_blocks(_i(3), _i(3), _i(3, 4), _i(9), _i(1), 9, _i(5), _i(4), _i(3), _i(1), _i(3))
    with pytest.raises(ValueError, match="suffix_lens holds 2"):
        pcr._ints(cpu, 3, _i(2), "suffix_lens")
    with pytest.raises(ValueError, match="block_tables must be"):
        pcr.assign_blocks(_i(3), _i(3), _i(12), _i(9), _i(1), 9, _i(5), _i(4), _i(3), _i(1), _i(3))
    with pytest.raises(ValueError, match="block_tables must be"):
        pcr.release_blocks(_i(2), _i(2), _i(4), _i(4), _i(1), 4, _i(1), _i(3))
    with pytest.raises(ValueError, match="current GPU"):
        pcr.release_blocks(_i(2), _i(2), _i(2, 4), _i(4), _i(1), 4, _i(1), _i(3))


def _h(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def test_binding_rows():
    gpu = (torch, -1)                                    # a CPU tensor's index
    assert pcr._rows(gpu, _h(5, 2, 64), 5, 2, 64, "x") == 128
    assert pcr._rows(gpu, _h(5, 128), 5, 2, 64, "x") == 128
    assert pcr._rows(gpu, _h(5, 300)[:, 44:172], 5, 2, 64, "x") == 300
    assert pcr._rows(gpu, _h(1, 300)[:, 44:172], 1, 2, 64, "x") == 128
    for x, msg in ((_h(4, 2, 64), "must be"), (torch.zeros(5, 2, 64), "2-byte"), (_h(5, 64, 2).transpose(1, 2), "back to back"),
                   (_h(5, 2, 128)[:, :, :64], "back to back"), (_h(2, 5, 64).transpose(0, 1), "back to back")):
        with pytest.raises(ValueError, match=msg):
            pcr._rows(gpu, x, 5, 2, 64, "x")
    with pytest.raises(ValueError, match="current GPU"):
        pcr._rows((torch, 0), _h(5, 2, 64), 5, 2, 64, "x")
    assert pcr._positions(gpu, _i(3, 9)[:, :5], 3, 5) == 9 and pcr._positions(gpu, _i(5), 1, 5) == 5
    for x, msg in ((_i(2, 5), "must be"), (_i(5), "must be"), (torch.zeros(3, 5, dtype=torch.int64), "int64"),
                   (_i(5, 3).t(), "back to back"), (_i(1, 5).expand(3, 5), "overlap")):
        with pytest.raises(ValueError, match=msg):
            pcr._positions(gpu, x, 3, 5)
    with pytest.raises(ValueError, match="length"):
        pcr.Rope(np.ones(8), np.zeros(7))


def test_binding_cross_and_append():
    pool = pcr.KVPool(_h(4, 2, 1024), _h(4, 2, 1024), 2, 64)
    n, cu = np.array([5, 9], np.int32), np.array([0, 1, 3], np.int32)
    with pytest.raises(ValueError, match="B\\+1"):
        pcr.cross_attn(_h(3, 4, 64), pool, _i(2, 4), _i(2), _i(3), n, cu[:2], 4, _h(3, 4, 64))
    with pytest.raises(ValueError, match="q holds 512"):
        pcr.cross_attn(_h(2, 4, 64), pool, _i(2, 4), _i(2), _i(3), n, cu, 4, _h(3, 4, 64))
    with pytest.raises(ValueError, match="current GPU"):
        pcr.cross_attn(_h(3, 4, 64), pool, _i(2, 4), _i(2), _i(3), n, cu, 4, _h(3, 4, 64))
    with pytest.raises(ValueError, match="pool.v holds"):
        pcr._pool_here((torch, -1), pcr.KVPool(_h(4, 2, 1024), _h(3, 2, 1024), 2, 64))
    rope = pcr.Rope(np.ones(32))
    with pytest.raises(ValueError, match="current GPU"):
        pcr.rope_append_kv(rope, pool, _h(5, 4, 64), _h(5, 2, 64), _h(5, 2, 64), _i(5), _i(5), 4, _h(5, 4, 64))
