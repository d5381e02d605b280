"""GPU: cross attention over an encoder's cached states against softmax attention in 64 bits.

Tolerance per element, from the rounding points: the weights enter the product with V rounded to
bf16 (relative 2^-8 each) and are normalised by the sum of the rounded values, which moves the
output by at most 2^-8 / (1 - 2^-8) * sum_j w_j |v_j - out| (computed beside the reference);
fp32 scores, exp2 and sums add less than a quarter of that at these magnitudes (|score| < 64:
2^-24 * 128 * 64 = 2^-11 relative); the output's own rounding is 2^-8 of its value."""
import numpy as np
import pytest
import torch

import opref
from paper_2603_23049_amd import pcr

pytestmark = pytest.mark.gpu
BS = 16


def _case(keys, rows, Hq, Hkv, d, seed, q_scale=1.0, poison=True, shared=False):
    rng = np.random.Generator(np.random.PCG64(seed))
    gen = torch.Generator().manual_seed(seed)
    blocks = [-(-n // BS) for n in keys]
    nb = sum(blocks) + 3
    perm = rng.permutation(nb).astype(np.int32)
    bt = np.full((len(keys), max(blocks + [1]) + 1), -1, np.int32)
    at = 0
    for b, n in enumerate(blocks):
        bt[b, :n] = perm[at:at + n]
        at += n
    if shared:
        bt[1:] = bt[0]
    pk = torch.randn(nb, Hkv, BS * d, generator=gen).to(torch.bfloat16)
    pv = torch.randn(nb, Hkv, BS * d, generator=gen).to(torch.bfloat16)
    if poison and not shared:                 # slots past each sequence's end: NaN and infinities
        kv, vv = pk.view(nb, Hkv, BS, d), pv.view(nb, Hkv, d, BS)
        for b, n in enumerate(keys):
            if n % BS:
                kv[bt[b, n // BS], :, n % BS:] = float("nan")
                vv[bt[b, n // BS], :, :, n % BS:] = float("inf") if b % 2 else float("nan")
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    q = (q_scale * torch.randn(int(cu[-1]), Hq, d, generator=gen)).to(torch.bfloat16)
    return q, pk, pv, bt, np.array(keys, np.int32), cu


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _run(q, pk, pv, bt, n, cu, Hkv, d, sm_scale=None, tail=5, stream=None, workspace=None):
    T, Hq = int(cu[-1]), q.shape[1]
    pool = pcr.KVPool(pk.cuda(), pv.cuda(), Hkv, d)
    out = torch.full((T + tail, Hq, d), 9.0, dtype=torch.bfloat16, device="cuda")
    pcr.cross_attn(q.cuda(), pool, _dev(bt), _dev(n), _dev(cu), n, cu, Hq, out, workspace=workspace, sm_scale=sm_scale,
                   stream=stream)
    torch.cuda.synchronize()
    assert (out[T:] == 9).all(), "rows behind the last sequence"
    return out[:T].cpu()


def _close(got, q, pk, pv, bt, n, cu, Hkv, d, sm_scale=None):
    want, dev = opref.cross(q.double(), pk.double(), pv.double(), bt, n, cu, Hkv, sm_scale or d ** -0.5)
    assert torch.isfinite(got.float()).all()
    err = (got.double() - want).abs()
    tol = 1.25 * dev * 2.0 ** -8 / (1 - 2.0 ** -8) + want.abs() * 2.0 ** -8 + 1e-30
    assert (err <= tol).all(), (float((err - tol).max()), float(err.max()))


@pytest.mark.parametrize("keys,rows,Hq,Hkv,d", [
    ([1], [1], 8, 8, 64), ([16], [1], 8, 1, 128), ([17], [3], 4, 4, 64), ([100, 1, 0, 33], [1, 1, 1, 1], 32, 8, 128),
    ([1500], [5], 16, 16, 64), ([0], [4], 8, 2, 64), ([0, 40], [0, 2], 4, 2, 128), ([1601, 3000, 31], [1, 1, 1], 16, 2, 128),
    ([257, 64, 65, 0, 1], [33, 70, 1, 6, 129], 8, 2, 64), ([700, 90], [300, 41], 14, 2, 128), ([63, 64, 65], [32, 64, 257], 8, 8, 128),
    ([500], [9], 40, 2, 64), ([2000, 10], [4, 16], 24, 1, 128), ([333], [1], 64, 2, 64), ([129, 800], [2, 4], 32, 8, 64),
    ([4000], [130], 8, 1, 128), ([2500, 77], [260, 1], 4, 4, 64)])
def test_equals_softmax_attention(keys, rows, Hq, Hkv, d):
    c = _case(keys, rows, Hq, Hkv, d, sum(keys) + sum(rows) + d)
    _close(_run(*c, Hkv, d), *c, Hkv, d)


@pytest.mark.parametrize("rows", [[1, 2, 40], [1, 1, 1]])
@pytest.mark.parametrize("q_scale,sm_scale", [(0.0, None), (4.0, None), (1.0, 1e-3), (1.0, 0.5)])
def test_softmax_sharpness(rows, q_scale, sm_scale):
    c = _case([300, 45, 1000], rows, 8, 2, 64, 17, q_scale)
    _close(_run(*c, 2, 64, sm_scale), *c, 2, 64, sm_scale)


def test_many_sequences():
    rng = np.random.Generator(np.random.PCG64(6))
    keys = rng.integers(0, 90, size=300).tolist()
    rows = rng.integers(0, 4, size=300).tolist()
    c = _case(keys, rows, 4, 2, 64, 8)
    _close(_run(*c, 2, 64), *c, 2, 64)
    rows = [1] * 300
    c = _case(keys, rows, 4, 2, 64, 8)
    _close(_run(*c, 2, 64), *c, 2, 64)


def test_shared_blocks_and_beams_give_the_same_rows():
    """Beams as rows of one sequence, and as sequences that share the blocks: the same values to
    the tolerance; and each repeats bit for bit."""
    q, pk, pv, bt, n, cu = _case([600] * 4, [1] * 4, 16, 4, 128, 3, poison=False, shared=True)
    a = _run(q, pk, pv, bt, n, cu, 4, 128)
    one = (q, pk, pv, bt[:1], n[:1], np.array([0, 4], np.int32))
    b = _run(*one, 4, 128)
    _close(a, q, pk, pv, bt, n, cu, 4, 128)
    _close(b, *one, 4, 128)
    assert torch.equal(a, _run(q, pk, pv, bt, n, cu, 4, 128)) and torch.equal(b, _run(*one, 4, 128))


def test_block_ids_do_not_change_the_bits():
    q, pk, pv, bt, n, cu = _case([500, 170], [3, 150], 8, 2, 64, 4)
    a = _run(q, pk, pv, bt, n, cu, 2, 64)
    nb = pk.shape[0]
    perm = torch.randperm(nb, generator=torch.Generator().manual_seed(1))
    inv = torch.empty_like(perm)
    inv[perm] = torch.arange(nb)
    bt2 = np.where(bt >= 0, inv.numpy()[bt.clip(0)], 2 ** 31 - 1).astype(np.int32)
    assert torch.equal(a, _run(q, pk[perm], pv[perm], bt2, n, cu, 2, 64))


@pytest.mark.parametrize("keys,rows,Hq,Hkv,d", [([3000, 40, 0], [1, 1, 1], 8, 2, 64), ([900, 2000], [70, 5], 16, 2, 128),
                                                ([5000], [20], 8, 1, 128)])
def test_streams_and_graph_replays(keys, rows, Hq, Hkv, d):
    c = _case(keys, rows, Hq, Hkv, d, 12)
    q, pk, pv, bt, n, cu = c
    want = _run(*c, Hkv, d)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    assert torch.equal(_run(*c, Hkv, d, stream=st), want)
    pool = pcr.KVPool(pk.cuda(), pv.cuda(), Hkv, d)
    nbytes = pcr.cross_attn_workspace_bytes(len(keys), int(cu[-1]), Hq, Hkv, d, max(keys))
    ws = torch.full((max(nbytes, 16),), 255, dtype=torch.uint8, device="cuda")
    args = (q.cuda(), pool, _dev(bt), _dev(n), _dev(cu), n, cu, Hq)
    out = torch.zeros_like(args[0])
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        pcr.cross_attn(*args, out, workspace=ws)
    for i in range(3):
        out.fill_(float("nan"))
        ws.fill_(255)                       # NaN bit patterns: nothing is read that the call did not write
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), want), i
        eager = torch.zeros_like(out)
        pcr.cross_attn(*args, eager, workspace=ws)
        assert torch.equal(eager.cpu(), want)
