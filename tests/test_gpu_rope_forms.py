"""GPU: the rotation's forms that take large calls: the tiles of the fused append at 64 and 128
dims, halves and adjacent pairs, heads turned whole and in part, with and without Q; and plain rows
whose workgroups walk several heads. Against the rotation in 64 bits, with test_gpu_rope's
tolerance, and bit for bit against the same tokens in calls small enough for the other forms."""
import numpy as np
import pytest
import torch

from paper_2603_23049_amd import pcr
from test_gpu_rope import _append_case, _bf16, _close, _gen, _positions, _rotation

pytestmark = pytest.mark.gpu
BS = 16
ROWS_BYTES = 4 << 20         # K and Q of a call that runs as rows of single waves, at most


@pytest.mark.parametrize("T,Hq,Hkv,d,rd,axes,interleaved,fused,bad", [
    (1733, 16, 4, 64, 64, 1, 0, 1, (0, 1, 40)), (1733, 16, 4, 64, 32, 3, 0, 0, (1732,)), (1701, 16, 4, 64, 64, 2, 1, 0, ()),
    (1750, 16, 8, 64, 48, 4, 1, 1, (3, 800, 801)), (17000, 1, 1, 64, 16, 1, 0, 0, ()), (960, 16, 2, 128, 128, 1, 1, 1, (7,)),
    (951, 16, 2, 128, 64, 3, 1, 0, ()), (977, 14, 7, 128, 32, 2, 0, 1, (976, 5)), (955, 16, 16, 128, 112, 4, 0, 0, ()),
    (2201, 0, 8, 128, 128, 1, 0, 1, (2,)), (2099, 0, 8, 128, 64, 2, 1, 0, ()), (4201, 0, 8, 64, 64, 3, 1, 1, (4200,))])
def test_append_tiles(T, Hq, Hkv, d, rd, axes, interleaved, fused, bad):
    assert T * (Hq + Hkv) * d * 2 > ROWS_BYTES
    c = _append_case(T, Hq, Hkv, d, rd, axes, interleaved, fused, 10 ** 6, T + rd, bad)
    pos, slots = c["pos"].cuda(), torch.from_numpy(c["slots"].astype(np.int32)).cuda()

    def run(cuts):
        pool = pcr.KVPool(c["pk"].cuda(), c["pv"].cuda(), Hkv, d)
        out = torch.full((T + 1, Hq, d), 3.0, dtype=torch.bfloat16, device="cuda")
        for a, b in zip(cuts, cuts[1:]):
            pcr.rope_append_kv(c["rope"], pool, c["qd"][a:b] if Hq else None, c["kd"][a:b], c["vd"][a:b], pos[:, a:b],
                               slots[a:b], Hq, out[a:b] if Hq else None)
        torch.cuda.synchronize()
        assert (out[T:] == 3).all()
        return out[:T], pool

    out, pool = run([0, T])
    step = ROWS_BYTES // ((Hq + Hkv) * d * 2) // 3
    small, spool = run([*range(0, T, step), T])            # every part runs as rows
    assert torch.equal(out, small) and torch.equal(pool.k, spool.k) and torch.equal(pool.v, spool.v)
    if Hq:
        _close(out, c["q"], c["pos"], c["f"], c["axis"], interleaved)
        assert torch.equal(out[:, :, rd:].cpu(), c["q"][:, :, rd:])
    live = (c["slots"] >= 0) & (c["slots"] < c["nb"] * BS)
    blk, o = torch.from_numpy(c["slots"][live] // BS), torch.from_numpy(c["slots"][live] % BS)
    k_got = pool.k.cpu().view(c["nb"], Hkv, BS, d)
    _close(k_got[blk, :, o], c["k"][live], c["pos"][:, live], c["f"], c["axis"], interleaved)
    want_v = c["pv"].clone().view(c["nb"], Hkv, d, BS)
    want_v[blk, :, :, o] = c["v"][live]
    assert torch.equal(pool.v.cpu().view(torch.int16), want_v.view(c["nb"], Hkv, BS * d).view(torch.int16))
    rest = torch.ones(c["nb"], BS, dtype=torch.bool)
    rest[blk, o] = False
    old = c["pk"].view(c["nb"], Hkv, BS, d).permute(0, 2, 1, 3)[rest]
    assert torch.equal(k_got.permute(0, 2, 1, 3)[rest].contiguous().view(torch.int16), old.contiguous().view(torch.int16))


@pytest.mark.parametrize("T,H,d,rd,axes,interleaved", [
    (5003, 16, 64, 64, 1, 1), (4101, 18, 80, 48, 2, 1), (2111, 17, 128, 128, 3, 1), (2100, 19, 128, 32, 4, 0),
    (5003, 13, 64, 64, 1, 0), (1300, 23, 256, 96, 3, 1), (9000, 9, 48, 48, 2, 0)])
@pytest.mark.parametrize("inverse", [False, True])
def test_rows_of_several_heads(T, H, d, rd, axes, interleaved, inverse):
    """The workgroups take four heads each from 256 of them on; fewer than that, of as many tokens
    as a part of the call has, take one."""
    per = 256 // (d // 16)
    assert -(-T // per) * -(-H // 4) >= 256
    gen = _gen(T + rd)
    x, pos = _bf16(gen, T, H, d), _positions(gen, axes, T, 10 ** 6)
    f, axis = _rotation(rd, axes, T)
    rope = pcr.Rope(f, axis, axes, bool(interleaved))
    xd, pd = x.cuda(), pos.cuda()
    out = torch.full((T + 2, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
    pcr.rope_rows(rope, xd, pd, out[1:T + 1], inverse=inverse)
    _close(out[1:T + 1], x, pos, f, axis, interleaved, inverse=inverse)
    assert (out[0] == 7).all() and (out[T + 1] == 7).all()
    assert torch.equal(out[1:T + 1, :, rd:].cpu(), x[:, :, rd:])
    small, step = torch.empty_like(xd), per * max(1, 200 // -(-H // 4)) // 2
    for a in range(0, T, step):
        pcr.rope_rows(rope, xd[a:a + step], pd[:, a:a + step], small[a:a + step], inverse=inverse)
    assert torch.equal(small, out[1:T + 1])
    pcr.rope_rows(rope, xd, pd, xd, inverse=inverse)
    assert torch.equal(xd, small)
