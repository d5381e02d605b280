"""GPU: cross attention of few rows where its work is cut in each of the ways the plan knows:
whole pairs with one to eight waves, parts of a pair, even runs over all pairs (runs that hold
several pairs, pairs that lie in many runs, more sequences than one wave scans), sequences
without rows or keys between them. The tolerance is test_gpu_cross's."""
import numpy as np
import pytest
import torch

from gpuio import attn_schedule
from test_gpu_cross import _case, _close, _run

pytestmark = pytest.mark.gpu


def _lens(n, lo, hi, seed, zeros=0):
    rng = np.random.Generator(np.random.PCG64(seed))
    v = rng.integers(lo, hi + 1, size=n)
    v[rng.integers(0, n, size=zeros)] = 0
    v[int(rng.integers(n))] = hi
    return v.tolist()


@pytest.mark.parametrize("keys,rows,Hq,Hkv,d", [
    (_lens(60, 20, 3000, 1), [1] * 60, 4, 1, 128),                         # even runs, single waves
    (_lens(130, 20, 3000, 2, 20), _lens(130, 0, 2, 3, 30), 2, 1, 128),     # the same, more than 64 sequences, gaps
    (_lens(40, 100, 6000, 4), [1] * 40, 4, 4, 64),                         # the same, 64 dims
    ([13000, 2000, 1000], [1, 1, 1], 8, 8, 128),                           # even runs of four waves
    ([2438, 2438], [1, 2], 14, 2, 128), ([9000], [4], 4, 1, 64),           # parts of a pair
    (_lens(30, 1, 500, 5), [1] * 30, 8, 8, 64), (_lens(9, 1, 90, 6, 2), [2] * 9, 4, 2, 128),   # whole pairs
    (_lens(300, 1, 200, 7, 40), _lens(300, 0, 3, 8, 50), 8, 4, 64), (_lens(300, 30, 60, 9), [1] * 300, 8, 8, 128),
    (_lens(300, 30, 90, 11), [1] * 300, 2, 1, 128), (_lens(300, 300, 700, 12), [1] * 300, 4, 4, 64),   # two waves; four
    (_lens(70, 1000, 2600, 10), [1] * 70, 16, 1, 128),                     # sixteen columns
])
def test_cuts(keys, rows, Hq, Hkv, d):
    c = _case(keys, rows, Hq, Hkv, d, len(keys) + d)
    got = _run(*c, Hkv, d)
    _close(got, *c, Hkv, d)
    assert torch.equal(got, _run(*c, Hkv, d))


def test_smaller_workspace_is_refused_and_a_batch_without_cuts_needs_none():
    from paper_2603_23049_amd import pcr
    q, pk, pv, bt, n, cu = _case([9000], [4], 4, 1, 64, 1)
    with pytest.raises(pcr.PcrError, match="needs a workspace"):
        _run(q, pk, pv, bt, n, cu, 1, 64, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    c = _case([40] * 20, [1] * 20, 8, 2, 64, 1)
    _close(_run(*c, 2, 64, workspace=torch.empty(0, dtype=torch.uint8, device="cuda")), *c, 2, 64)


def test_workspace_size_covers_smaller_batches():
    from paper_2603_23049_amd import pcr
    big = pcr.cross_attn_workspace_bytes(64, 64, 8, 2, 128, 9000)
    for B, T, n in ((1, 1, 9000), (3, 3, 8999), (64, 64, 100), (40, 41, 5000), (2, 60, 9000)):
        assert pcr.cross_attn_workspace_bytes(B, T, 8, 2, 128, n) <= big
    for keys, rows in (([9000], [1]), ([9000, 1, 5000], [1, 1, 2]), ([4000] * 64, [1] * 64)):
        c = _case(keys, rows, 8, 2, 128, 5, poison=False, shared=True)
        q, pk, pv, bt, n, cu = c
        _run(q, pk, pv, bt, n, cu, 2, 128, workspace=torch.empty(big, dtype=torch.uint8, device="cuda"))


def test_workspace_size_with_sequences_without_rows():
    """Two of 64 sequences have a row: the size for 2 rows in all serves a plan of parts of all 64."""
    c = _case([800, 800] + [0] * 62, [1, 1] + [0] * 62, 1, 1, 64, 2)
    _close(_run(*c, 1, 64), *c, 1, 64)


@pytest.mark.parametrize("schedule", ["key_halves", "row_halves"])
@pytest.mark.parametrize("keys,rows,Hq,Hkv,d", [([65, 0, 300], [70, 3, 150], 8, 2, 64), ([129, 1000], [33, 1], 8, 1, 128),
                                                ([640], [600], 2, 1, 128)])
def test_row_tile_schedules(schedule, keys, rows, Hq, Hkv, d):
    c = _case(keys, rows, Hq, Hkv, d, 31)
    with attn_schedule(schedule):
        _close(_run(*c, Hkv, d), *c, Hkv, d)


@pytest.mark.parametrize("keys,rows,Hq,Hkv,d", [
    ([6000, 7000], [20, 1], 8, 1, 128), ([5000, 100, 6400, 0], [17, 40, 2, 3], 4, 1, 64),   # keys of row tiles and few rows cut
    (_lens(140, 1, 100, 13, 9), [20] * 140, 2, 2, 64)])                                # more sequences than one launch's map
def test_row_tiles(keys, rows, Hq, Hkv, d):
    c = _case(keys, rows, Hq, Hkv, d, 32)
    got = _run(*c, Hkv, d)
    _close(got, *c, Hkv, d)
    assert torch.equal(got, _run(*c, Hkv, d))
