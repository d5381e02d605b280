"""GPU: kept tokens moved into consecutive slots of every layer, bit for bit."""
import numpy as np
import pytest
import torch

import treeref
from paper_2603_23049_amd import pcr
from gpuio import dev, u16

pytestmark = pytest.mark.gpu
BS = 16


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


def _case(p, reach, Hkv, d, L, seed, width=None):
    """Pools of L layers and tables for sequences of p tokens with `reach` positions after them."""
    rng = np.random.Generator(np.random.PCG64(seed))
    blocks = [-(-(a + r) // BS) for a, r in zip(p, reach)]
    nb = sum(blocks) + 2
    perm = rng.permutation(nb)
    bt = np.full((len(p), width or max(blocks)), -1, np.int32)
    at = 0
    for b, k in enumerate(blocks):
        bt[b, :k] = perm[at:at + k]
        at += k
    kv = rng.integers(0, 2 ** 16, size=(L, 2, nb, Hkv, BS * d)).astype(np.uint16)     # any bits, NaN among them
    return rng, bt, kv


def _check(kv, bt, p, path, kept, Hkv, d, stream=None):
    t = [[dev(layer[0]), dev(layer[1])] for layer in kv]
    pools = pcr.KVLayers([pcr.KVPool(a, b, Hkv, d) for a, b in t])
    args = _i32(bt), _i32(p), _i32(path), _i32(kept)
    torch.cuda.synchronize()
    pcr.compact_kv(pools, *args, stream=stream)
    torch.cuda.synchronize()
    for layer, (a, b) in zip(kv, t):
        wk, wv = treeref.compact(layer[0], layer[1], bt, p, path, kept)
        assert np.array_equal(u16(a), wk) and np.array_equal(u16(b), wv)


def _paths(rng, n, cap):
    path = np.full((len(n), cap), -1, np.int32)
    kept = np.zeros(len(n), np.int32)
    for b, s in enumerate(n):
        kept[b] = k = int(rng.integers(0, min(s, cap) + 1))
        path[b, :k] = np.sort(rng.permutation(s)[:k])
    return path, kept


@pytest.mark.parametrize("Hkv,d,L", [(1, 64, 1), (3, 64, 2), (8, 128, 3), (5, 128, 1), (2, 64, 130)])
@pytest.mark.parametrize("p,n,cap", [([0], [1], 1), ([15], [3], 3), ([0, 7, 31], [20, 9, 64], 12), ([100, 3], [200, 40], 150),
                                     ([16, 17, 14, 0], [1, 2, 5, 17], 8)])
def test_paths(p, n, cap, Hkv, d, L):
    rng, bt, kv = _case(p, n, Hkv, d, L, sum(p) + sum(n) + L)
    for _ in range(2):
        path, kept = _paths(rng, n, cap)
        _check(kv, bt, p, path, kept, Hkv, d)


def test_every_way_of_a_block():
    """One source and one target slot after another, over block ends."""
    p, n = [11], [40]
    rng, bt, kv = _case(p, n, 2, 64, 1, 3)
    for first in range(0, 24, 5):
        path = np.arange(first, first + 16)[None, :]
        _check(kv, bt, p, path, [16], 2, 64)
    _check(kv, bt, p, np.array([[0, 2, 3, 4, 5, 6, 7, 8, 9, 39]]), [10], 2, 64)      # sources that are targets
    _check(kv, bt, p, np.arange(1, 40)[None, :], [39], 2, 64)


def test_paths_that_end_the_moves():
    p, n = [5, 5, 5, 5, 5, 5, -1, 5], [60] * 8
    rng, bt, kv = _case([5] * 8, n, 2, 128, 2, 4)
    path = np.tile(np.array([[1, 3, 4, 9, 12, 20, 30, 31, 40, 50]]), (8, 1))
    kept = np.array([10, 99, 0, -3, 10, 10, 10, 10])
    path[0, 5] = 12                      # not ascending
    path[4, 9] = 10 ** 6                 # past the table's row
    path[5, 2] = -1
    path[7, 0] = -5
    _check(kv, bt, p, path, kept, 2, 128)
    bt2 = bt.copy()
    bt2[0, 2], bt2[1, 0], bt2[4, 1] = -1, 10 ** 6, -7
    _check(kv, bt2, p, path, kept, 2, 128)
    path[4, 9] = 2 ** 31 - 1             # the position's sum does not wrap
    _check(kv, bt2, p, path, kept, 2, 128)


def test_stream_and_graph():
    p, n = [9, 30], [30, 12]
    rng, bt, kv = _case(p, n, 4, 64, 3, 5)
    path, kept = np.array([[0, 2, 9, 20], [3, 4, 8, -1]]), np.array([4, 3])
    s = torch.cuda.Stream()
    _check(kv, bt, p, path, kept, 4, 64, stream=s)
    t = [[dev(layer[0]), dev(layer[1])] for layer in kv]
    pools = pcr.KVLayers([pcr.KVPool(a, b, 4, 64) for a, b in t])
    args = _i32(bt), _i32(p), _i32(path), _i32(kept)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pcr.compact_kv(pools, *args)
    want = [(layer[0], layer[1]) for layer in kv]
    for _ in range(3):                   # each replay moves what the one before left
        g.replay()
        torch.cuda.synchronize()
        want = [treeref.compact(k, v, bt, p, path, kept) for k, v in want]
        for (wk, wv), (a, b) in zip(want, t):
            assert np.array_equal(u16(a), wk) and np.array_equal(u16(b), wv)
