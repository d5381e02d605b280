"""GPU: draft trees and tree attention against their definitions in 64 bits, at the sizes and
masks where they can go wrong."""
import numpy as np
import pytest
import torch

import treeref
from paper_2603_23049_amd import pcr

pytestmark = pytest.mark.gpu
BS = 16


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


def _words(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int64)).cuda()


@pytest.mark.parametrize("n,words", [([1], 1), ([64], 1), ([65, 0, 3], 2), ([5, 300, 128, 1], 5), ([1000], 16), ([70], 1)])
def test_draft_tree(n, words):
    rng = np.random.Generator(np.random.PCG64(sum(n) + words))
    B, cu = len(n), np.concatenate([[0], np.cumsum(n)])
    parents = np.concatenate([np.array(treeref.random_parents(rng, s), np.int32) for s in n])
    T = len(parents) + 5                                # rows behind the last sequence
    parents = np.concatenate([parents, np.full(5, -1, np.int32)])
    for t in rng.integers(0, T - 5, size=(T - 5) // 9):   # padding, and parents that no node can have
        parents[t] = rng.choice([-1, -2, 10 ** 9, -2 ** 31, 2 ** 31 - 1, t])
    p = rng.integers(0, 100000, size=B)
    vis, pos = rng.integers(0, 2 ** 63, size=(T, words)).astype(np.uint64), rng.integers(0, 99, size=T).astype(np.int32)
    want = treeref.draft_tree(cu, parents, p, T, words, vis, pos)
    v, q = _words(vis), _i32(pos)
    pcr.draft_tree(_i32(cu), _i32(parents), _i32(p), v, q)
    assert np.array_equal(v.cpu().numpy().view(np.uint64), want[0])
    assert np.array_equal(q.cpu().numpy(), want[1])


class Case:
    """Sequences of p cached tokens and n nodes, with a pool, tables and random trees."""

    def __init__(self, p, n, Hq, Hkv, d, words=1, seed=1, scale_q=1.0, pad=3):
        rng = np.random.Generator(np.random.PCG64(seed))
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.p, self.n, self.Hq, self.Hkv, self.d, self.words = np.array(p, np.int32), np.array(n, np.int32), Hq, Hkv, d, words
        self.cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        self.T = int(self.cu[-1])
        blocks = -(-(self.p + self.n) // BS)
        nb = int(blocks.sum()) + 3
        perm = rng.permutation(nb)
        self.bt = np.full((len(p), max(1, int(blocks.max()))), -1, np.int32)
        at = 0
        for b, k in enumerate(blocks):
            self.bt[b, :k] = perm[at:at + k]
            at += k
        self.spare = perm[at:]
        rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)      # noqa: E731
        self.k, self.v = rand(nb, Hkv, BS * d), rand(nb, Hkv, BS * d)
        self.q = (rand(self.T + pad, Hq, d) * scale_q).contiguous()
        self.parents = np.concatenate([np.array(treeref.random_parents(rng, int(s)), np.int32) for s in n])
        self.visible = treeref.words_of(self.cu, self.parents, words)
        self.scale = 1.0 / d ** 0.5
        self.pad = pad

    def run(self, **kw):
        out = torch.full_like(self.q, 7.0)
        pcr.tree_attn(self.q, pcr.KVPool(self.k, self.v, self.Hkv, self.d), _i32(self.bt), _i32(self.p), _i32(self.cu),
                      self.p, self.cu, _words(self.visible), self.Hq, out, sm_scale=self.scale, **kw)
        return out

    def want(self):
        return treeref.tree_attn(self.q[:self.T].cpu().double(), self.k.cpu().double(), self.v.cpu().double(), self.bt,
                                 self.p, self.cu, self.visible, self.Hkv, self.scale)

    def check(self, out=None):
        out = self.run() if out is None else out
        torch.cuda.synchronize()
        want, dev = self.want()
        got = out[:self.T].cpu().double()
        # Weights rounded to bf16 (each off by 2^-8 of itself at most, numerator and sum) move a row by at
        # most 2^-8 / (1 - 2^-8) of sum w |v - out|; a quarter more covers fp32 scores and sums; the
        # result is rounded to bf16.
        tol = 1.25 * dev * 2.0 ** -8 / (1 - 2.0 ** -8) + want.abs() * 2.0 ** -8 + 1e-30
        err = (got - want).abs()
        assert (err <= tol).all(), (float((err - tol).max()), int((err > tol).sum()))
        assert (out[self.T:] == 7.0).all()


HEADS = [(8, 8, 64), (8, 2, 128), (28, 4, 128), (16, 1, 64), (64, 2, 128)]


@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
@pytest.mark.parametrize("p,n,words", [
    ([0], [1], 1), ([1], [1], 1), ([15, 16, 17], [1, 1, 1], 1), ([31], [2], 1), ([100], [8], 1),
    ([0, 0], [64, 7], 1), ([5, 250, 0, 33], [16, 0, 3, 64], 1), ([40, 3], [65, 130], 3), ([1000, 77], [13, 21], 1),
    ([24, 8], [5, 61], 2)])
def test_sizes(p, n, words, Hq, Hkv, d):
    Case(p, n, Hq, Hkv, d, words, seed=sum(p) + sum(n) + d).check()


@pytest.mark.parametrize("scale_q", [0.0, 8.0, 32.0])
def test_sharp_rows(scale_q):
    Case([70, 300], [9, 33], 8, 2, 128, scale_q=scale_q).check()


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 64), (8, 1, 128), (28, 4, 128)])
@pytest.mark.parametrize("p", [0, 3, 40])
def test_any_words(Hq, Hkv, d, p):
    """Rows that see nothing of the tree, not themselves, every node, or bits past the last node."""
    c = Case([p, 0, 21], [50, 20, 70], Hq, Hkv, d, words=2, seed=p + d)
    rng = np.random.Generator(np.random.PCG64(p))
    c.visible = rng.integers(0, 2 ** 63, size=c.visible.shape).astype(np.uint64) * np.uint64(2)
    c.visible[::3] = 0
    c.visible[1::7] = np.uint64(2 ** 64 - 1)
    out = c.run()
    c.check(out)
    if p == 0:
        assert (out[0] == 0).all() and (out[c.cu[1]:c.cu[2]][(c.visible[c.cu[1]:c.cu[2]] == 0).all(1)] == 0).all()


def _slot(c, b, pos):
    return int(c.bt[b, pos // BS]), pos % BS


def _set(c, b, pos, k=None, v=None):
    blk, o = _slot(c, b, pos)
    if k is not None:
        c.k.view(-1, c.Hkv, BS, c.d)[blk, :, o] = k
    if v is not None:
        c.v.view(-1, c.Hkv, c.d, BS)[blk, :, :, o] = v


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("Hq,Hkv,d,n,p", [(8, 2, 64, 20, 37), (16, 2, 128, 40, 5), (8, 8, 64, 3, 100), (64, 2, 128, 64, 10)])
def test_hidden_values_do_not_reach_a_row(Hq, Hkv, d, n, p, bad):
    """Infinite and NaN K/V past the end, in blocks of nobody, and in a node that only it sees."""
    c = Case([p, 64], [n, n], Hq, Hkv, d, seed=n)
    want = c.run()
    leaf = [i for i in range(n) if i not in c.parents[:n]][-1]        # nobody's parent
    _set(c, 0, p + leaf, bad, bad)
    for b, last in enumerate(c.p + c.n):
        for pos in range(int(last), -(-int(last) // BS) * BS):
            _set(c, b, pos, bad, bad)
    c.k[torch.from_numpy(c.spare.copy()).cuda()] = bad
    c.v[torch.from_numpy(c.spare.copy()).cuda()] = bad
    out = c.run()
    rows = torch.arange(c.T) != leaf
    assert torch.equal(out[:c.T][rows].view(torch.int16), want[:c.T][rows].view(torch.int16))
    assert not torch.isfinite(out[leaf].float()).any()


@pytest.mark.parametrize("Hq,Hkv,d,n", [(8, 2, 64, 20), (16, 2, 128, 40), (64, 2, 128, 64)])
def test_seen_infinities_arrive(Hq, Hkv, d, n):
    """V's infinities and NaN of a seen node reach the rows that see it, in their dims alone."""
    c = Case([37], [n], Hq, Hkv, d, seed=n)
    c.visible[:] = 0
    for i in range(n):
        c.visible[i, 0] = 1 << i
    c.visible[n - 1, 0] = 0b1110                       # sees nodes 1, 2 and 3
    base = c.run()
    vv = c.v.view(-1, Hkv, d, BS)
    for node, dim, val in ((1, 3, float("inf")), (2, 9, -float("inf")), (3, 17, float("nan")), (1, 20, float("inf")),
                           (2, 20, -float("inf"))):
        blk, o = _slot(c, 0, 37 + node)
        vv[blk, :, dim, o] = val
    out = c.run()
    row, was = out[n - 1].float(), base[n - 1].float()
    assert (row[:, 3] == float("inf")).all() and (row[:, 9] == -float("inf")).all()
    assert torch.isnan(row[:, 17]).all() and torch.isnan(row[:, 20]).all()
    rest = [x for x in range(d) if x not in (3, 9, 17, 20)]
    assert torch.equal(row[:, rest], was[:, rest])
    others = [i for i in range(n - 1) if i not in (1, 2, 3)]
    assert torch.equal(out[others], base[others])


def test_ids_outside_the_pool():
    c = Case([40], [10], 8, 2, 64)
    c.bt[0, 1] = 10 ** 6
    out = c.run()
    c.bt[0, 1] = 0
    assert torch.equal(out, c.run())


def test_chain_is_prefill():
    """A chain sees what causal attention sees: both within their rounding of the same values."""
    c = Case([130, 17], [48, 5], 16, 2, 128)
    c.parents = np.concatenate([np.arange(s) - 1 for s in c.n]).astype(np.int32)
    c.visible = treeref.words_of(c.cu, c.parents, 1)
    out = c.run()
    c.check(out)
    ref = torch.zeros_like(out)
    pcr.prefix_prefill_attn(c.q, pcr.KVPool(c.k, c.v, 2, 128), _i32(c.bt), _i32(c.p), _i32(c.cu), c.p, c.cu, 16, ref)
    c.check(torch.cat([ref[:c.T], out[c.T:]]))


def test_same_bits_streams_and_graph():
    c = Case([900, 33, 0, 410], [16, 30, 4, 64], 32, 8, 128)
    want = c.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = c.run(stream=s)
    s.synchronize()
    assert torch.equal(want, other)
    pool, bt, p, cu, vis = pcr.KVPool(c.k, c.v, 8, 128), _i32(c.bt), _i32(c.p), _i32(c.cu), _words(c.visible)
    n = pcr.tree_attn_workspace_bytes(4, c.T, 32, 8, 128, int((c.p + c.n).max()))
    ws = torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
    out = torch.full_like(c.q, 7.0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pcr.tree_attn(c.q, pool, bt, p, cu, c.p, c.cu, vis, 32, out, workspace=ws, sm_scale=c.scale)
    for k in range(3):
        out.fill_(7.0)
        ws.fill_(255)
        c.q.copy_(c.q * (1.0 if k == 0 else 0.5))
        eager = c.run()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
