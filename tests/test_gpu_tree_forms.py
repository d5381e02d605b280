"""GPU: tree attention in every form that its work is cut in (which those are, test_tree_plan says on
the CPU): few rows as whole pairs, parts of a pair and even runs, row tiles by every schedule and
with their keys cut, with rows that see nothing of what a workgroup holds and hidden nodes that
hold infinities. The tolerance is test_gpu_tree's."""
import numpy as np
import pytest
import torch

from gpuio import attn_schedule
from paper_2603_23049_amd import pcr
from test_gpu_tree import Case, _i32, _set, _words

pytestmark = pytest.mark.gpu


def _spread(n, lo, hi, seed, first=None):
    v = np.random.Generator(np.random.PCG64(seed)).integers(lo, hi + 1, size=n).tolist()
    return [first or v[0]] + v[1:]


# p, nodes of each, Hq, Hkv, d: one tile of columns and two of each cut
FORMS = [
    ([1080], 9, 1, 1, 64), ([1080], 20, 1, 1, 64),                       # even runs, single waves
    ([545], 3, 4, 1, 128), ([545], 7, 4, 1, 128),
    ([12000] + [900] * 6, 2, 2, 1, 64), (_spread(5, 100, 998, 2, 13410), 5, 4, 1, 64),   # of four
    ([3840], 4, 1, 1, 128), ([6675], 9, 2, 1, 128),
    ([2080], 16, 1, 1, 64), ([2080], 8, 4, 1, 64), ([2080], 2, 8, 1, 128), ([2080], 4, 8, 1, 128),   # parts of a pair
    ([20], 5, 8, 8, 64), ([3], 17, 8, 8, 64), ([0], 5, 4, 2, 128), ([30], 9, 4, 2, 128),        # whole pairs, four waves
    (_spread(260, 1, 12, 3), 2, 4, 1, 64), (_spread(257, 0, 12, 4), 3, 8, 1, 64),
    (_spread(69, 0, 14, 5), 1, 16, 8, 64), (_spread(66, 0, 14, 6), 3, 64, 8, 64),             # two waves
    (_spread(34, 0, 14, 7), 2, 16, 8, 128), (_spread(33, 0, 14, 8), 3, 64, 8, 128),
    (_spread(131, 0, 14, 9), 2, 8, 8, 64), (_spread(141, 0, 10, 10), 5, 32, 8, 64),           # one
    (_spread(66, 0, 17, 11), 2, 8, 8, 128), (_spread(258, 0, 14, 12), 2, 32, 2, 128),
]


def _check(c):
    c.pad = 0
    out = c.run()
    c.check(out)
    assert torch.equal(out, c.run())


@pytest.mark.parametrize("p,n,Hq,Hkv,d", FORMS)
def test_few_rows(p, n, Hq, Hkv, d):
    _check(Case(p, [n] * len(p), Hq, Hkv, d, seed=len(p) + d + n))


@pytest.mark.parametrize("p,n,Hq,Hkv,d", [f for f in FORMS if len(f[0]) < 20])
def test_few_rows_that_see_nothing(p, n, Hq, Hkv, d):
    """Rows without a node, over the cached keys and (no cached keys, many nodes) over none."""
    c = Case(p + [0], [n] * len(p) + [n], Hq, Hkv, d, seed=3)
    c.visible[::2] = 0
    _check(c)


@pytest.mark.parametrize("schedule", ["auto", "key_halves", "row_halves"])
@pytest.mark.parametrize("p,n,Hq,Hkv,d,words", [
    ([65, 0, 300], [70, 3, 150], 8, 2, 64, 3), ([129, 1000], [33, 1], 8, 1, 128, 1), ([640], [200], 4, 2, 128, 4),
    ([5000], [40], 8, 1, 128, 1), ([6000, 0, 3000], [33, 60, 2], 4, 1, 64, 1)])     # the last two: keys cut
def test_row_tiles(schedule, p, n, Hq, Hkv, d, words):
    c = Case(p, n, Hq, Hkv, d, words, seed=sum(n))
    with attn_schedule(schedule):
        _check(c)
        c.visible[::3] = 0                               # rows of a tile that see its nodes, and rows that do not
        c.visible[5:40] = 0
        _check(c)


@pytest.mark.parametrize("schedule", ["auto", "key_halves", "row_halves"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("p,n,Hq,Hkv,d", [(5000, 40, 8, 1, 128), (70, 64, 8, 2, 64), (0, 64, 4, 1, 128), (1, 300, 2, 1, 64)])
def test_row_tiles_hidden_values(schedule, p, n, Hq, Hkv, d, bad):
    c = Case([p, 64], [n, 50], Hq, Hkv, d, words=-(-n // 64), seed=n)
    with attn_schedule(schedule):
        want = c.run()
        leaves = [i for i in range(n) if i not in c.parents[:n]]
        for i in leaves[::2]:
            _set(c, 0, p + i, bad, bad)
        for pos in range(p + n, -(-(p + n) // 16) * 16):
            _set(c, 0, pos, bad, bad)
        out = c.run()
    keep = torch.ones(c.T, dtype=torch.bool)
    keep[leaves[::2]] = False
    assert torch.equal(out[:c.T][keep].view(torch.int16), want[:c.T][keep].view(torch.int16))
    assert not torch.isfinite(out[:c.T][~keep].float()).any(-1).any()


@pytest.mark.parametrize("schedule", ["auto", "key_halves", "row_halves"])
@pytest.mark.parametrize("p,n,Hq,Hkv,d", [(5000, 40, 8, 1, 128), (37, 64, 8, 2, 64), (0, 130, 4, 1, 128),
                                             (2080, 8, 4, 1, 64), (6675, 4, 4, 1, 128), (1080, 20, 1, 1, 64)])
def test_seen_infinities(schedule, p, n, Hq, Hkv, d):
    """V's infinities and NaN of a seen node reach the rows that see it, in their dims alone."""
    c = Case([p], [n], Hq, Hkv, d, words=-(-n // 64), seed=n)
    c.visible[:] = 0
    for i in range(n):
        c.visible[i, i // 64] = np.uint64(1 << (i % 64))
    c.visible[n - 1] = 0
    c.visible[n - 1, 0] = 0b1110                         # sees nodes 1, 2 and 3
    with attn_schedule(schedule):
        base = c.run()
        vv = c.v.view(-1, Hkv, d, 16)
        for node, dim, val in ((1, 3, float("inf")), (2, 9, -float("inf")), (3, 17, float("nan")), (1, 20, float("inf")),
                               (2, 20, -float("inf"))):
            vv[int(c.bt[0, (p + node) // 16]), :, dim, (p + node) % 16] = val
        out = c.run()
    row, was = out[n - 1].float(), base[n - 1].float()
    assert (row[:, 3] == float("inf")).all() and (row[:, 9] == -float("inf")).all()
    assert torch.isnan(row[:, 17]).all() and torch.isnan(row[:, 20]).all()
    rest = [x for x in range(d) if x not in (3, 9, 17, 20)]
    assert torch.equal(row[:, rest], was[:, rest])
    others = [i for i in range(n - 1) if i not in (1, 2, 3)]
    assert torch.equal(out[others], base[others])


@pytest.mark.parametrize("n,Hq", [(5, 4), (40, 8)])
def test_a_row_of_nan_stays_alone(n, Hq):
    """A NaN query (a padding row, say) ends in its own row, in every form."""
    c = Case([100, 30], [n, n], Hq, 1, 128, seed=n)
    want = c.run()
    c.q[2] = float("nan")
    out = c.run()
    rows = torch.arange(c.T) != 2
    assert torch.equal(out[:c.T][rows].view(torch.int16), want[:c.T][rows].view(torch.int16))
    assert torch.isnan(out[2].float()).all()


def test_more_sequences_than_one_launch():
    rng = np.random.Generator(np.random.PCG64(5))
    _check(Case(rng.integers(0, 90, size=140).tolist(), rng.integers(0, 40, size=140).tolist(), 2, 2, 64, seed=9))


def test_workspace():
    c = Case([9000], [4], 4, 1, 64)
    with pytest.raises(pcr.PcrError, match="needs a workspace"):
        c.run(workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    c = Case([30], [40], 8, 2, 64)
    with pytest.raises(pcr.PcrError, match="needs a workspace"):
        c.run(workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    big = pcr.tree_attn_workspace_bytes(64, 640, 8, 2, 128, 9000)
    for B, T, n in ((1, 1, 9000), (3, 30, 8999), (64, 64, 100), (40, 410, 5000), (2, 600, 9000)):
        assert pcr.tree_attn_workspace_bytes(B, T, 8, 2, 128, n) <= big
    ws = torch.empty(big, dtype=torch.uint8, device="cuda")
    for p, n in (([8000], [1]), ([8000, 1, 5000], [4, 8, 1]), ([2000] * 20, [9] * 20)):
        Case(p, n, 8, 2, 128).check(Case(p, n, 8, 2, 128).run(workspace=ws))
    # two of 64 sequences have nodes: the size for 2 rows in all serves a plan of parts of all 64
    Case([800, 800] + [0] * 62, [1, 1] + [0] * 62, 1, 1, 64).check()


def test_two_calls_at_once():
    """Two streams, each call with its own workspace."""
    a, b = Case([3000, 40], [5, 3], 4, 1, 128, seed=1), Case([2000] * 3, [40] * 3, 8, 2, 128, seed=2)
    want = [a.run(), b.run()]
    args = [(pcr.KVPool(c.k, c.v, c.Hkv, c.d), _i32(c.bt), _i32(c.p), _i32(c.cu), c.p, c.cu, _words(c.visible)) for c in (a, b)]
    ws = [torch.empty(max(16, pcr.tree_attn_workspace_bytes(len(c.p), c.T, c.Hq, c.Hkv, c.d, int((c.p + c.n).max()))),
                      dtype=torch.uint8, device="cuda") for c in (a, b)]
    outs = [[torch.full_like(c.q, 7.0) for _ in range(20)] for c in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for k in range(20):
        for c, x, w, o, s in zip((a, b), args, ws, outs, streams):
            pcr.tree_attn(c.q, *x, c.Hq, o[k], workspace=w, sm_scale=c.scale, stream=s)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(x, w) for x in o)
