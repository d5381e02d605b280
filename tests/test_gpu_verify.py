"""GPU: verification of drafted tokens against its definition, whole numbers compared one by one."""
import numpy as np
import pytest
import torch

import treeref
from paper_2603_23049_amd import pcr

pytestmark = pytest.mark.gpu


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


def _softmax(x):
    e = np.exp(x - x.max(-1, keepdims=True))
    return (e / e.sum(-1, keepdims=True)).astype(np.float32)


class Case:
    def __init__(self, n, V, drawn, seed, back=4, cap=None, sharp=3.0, away=0.8):
        rng = np.random.Generator(np.random.PCG64(seed))
        self.n, self.V, self.B = np.array(n), V, len(n)
        self.cu = np.concatenate([[0], np.cumsum(n)])
        self.T = T = int(self.cu[-1])
        self.parents = np.concatenate([np.array(treeref.random_parents(rng, s, back), np.int32) for s in n] + [np.zeros(0, np.int32)])
        logits = sharp * rng.standard_normal((T, V))
        self.target = _softmax(logits)
        q = _softmax(0.97 * logits + away * rng.standard_normal((T, V)))
        self.tokens = np.zeros(T, np.int32)
        for b in range(self.B):
            used = {}
            for i in range(1, int(n[b])):
                t, u = int(self.cu[b]) + i, int(self.cu[b]) + int(self.parents[int(self.cu[b]) + i])
                if drawn:
                    self.tokens[t] = min(V - 1, np.searchsorted(np.cumsum(q[u].astype(np.float64)), rng.random()))
                else:
                    k = used[u] = used.get(u, -1) + 1
                    self.tokens[t] = np.argsort(-q[u], kind="stable")[k % V]
        self.draft = q if drawn else None
        self.uniforms = rng.random(T).astype(np.float32)
        self.uniforms[self.uniforms >= 1.0] = 0.5
        self.p = rng.integers(0, 5000, size=self.B)
        self.cap = cap or max(1, int(self.n.max()))

    def run(self, stride=0, in_place=False, extra=2):
        cuda = lambda a: torch.from_numpy(a).cuda()                  # noqa: E731

        def rows(a):
            if a is None:
                return None
            x = torch.full((self.T + extra, self.V + stride), float("nan"), device="cuda")
            x[:self.T, :self.V] = cuda(a)
            return x[:, :self.V]

        pad = lambda a: _i32(np.concatenate([a, np.full(extra, 3)]))      # noqa: E731
        B = self.B
        out = [torch.full((B + 1, self.cap), 77, dtype=torch.int32, device="cuda")] + \
              [torch.full((B + 1,), 77, dtype=torch.int32, device="cuda") for _ in range(3)]
        p = _i32(self.p)
        ctx = p if in_place else out[3][:B]
        pcr.verify_drafts(_i32(self.cu), pad(self.parents), pad(self.tokens), rows(self.target), rows(self.draft),
                          cuda(np.concatenate([self.uniforms, np.zeros(extra, np.float32)])), p, out[0][:B], out[1][:B],
                          out[2][:B], ctx)
        torch.cuda.synchronize()
        assert all((o[B:] == 77).all() for o in out)
        return [x.cpu().numpy() for x in (out[0][:B], out[1][:B], out[2][:B], ctx)]

    def want(self):
        return treeref.verify(self.cu, self.parents, self.tokens, self.target, self.draft, self.uniforms, self.p, self.cap)

    def check(self, **kw):
        got, want = self.run(**kw), self.want()
        for g, w, what in zip(got, want, ("path", "accepted_lens", "next_tokens", "context_lens")):
            assert np.array_equal(g, w), (what, g, w)
        return got


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("n,V,back", [
    ([1], 1, 1), ([1, 3], 2, 1), ([5], 63, 1), ([6, 1, 4], 64, 2), ([9, 0, 13], 65, 6), ([5] * 20, 1000, 1),
    ([25, 12, 3, 64], 4097, 6), ([8] * 40, 257, 8), ([70, 130], 333, 20), ([4, 4, 4], 33333, 1), ([9, 2], 131073, 8)])
def test_sizes(n, V, back, drawn):
    Case(n, V, drawn, sum(n) + V, back).check()


@pytest.mark.parametrize("drawn", [True, False])
def test_row_strides_in_place_and_short_paths(drawn):
    Case([9, 5, 30], 777, drawn, 5, 3).check(stride=3)
    Case([9, 5, 30], 777, drawn, 6, 3).check(in_place=True)
    for cap in (1, 2, 3):
        Case([9, 5, 30] * 5, 100, drawn, cap, 1, cap=cap, sharp=5.0, away=0.1).check()


def test_agreeing_draft_keeps_all():
    """q = p: every first child stays (u q < p), whole chains are kept."""
    c = Case([7] * 8, 500, True, 3, back=1)
    c.draft = c.target
    path, kept, _, _ = c.check()
    assert (kept == 7).all() and (path == np.arange(7)).all()


def test_certain_rows():
    """One-hot target rows (greedy decoding): the drafted token stays when it is the target's, and
    the drawn one is the target's whatever the random number."""
    rng = np.random.Generator(np.random.PCG64(8))
    for drawn in (True, False):
        c = Case([6] * 30, 50, drawn, 9, back=2)
        best = rng.integers(0, 50, size=c.T)
        c.target = np.zeros((c.T, 50), np.float32)
        c.target[np.arange(c.T), best] = 1.0
        for t in range(c.T):
            if rng.random() < 0.6 and c.parents[t] >= 0:
                c.tokens[t] = best[c.cu[t // 6] + c.parents[t]]
        c.uniforms[::5] = 0.0
        c.uniforms[1::5] = np.float32(1 - 2.0 ** -24)
        path, kept, nxt, _ = c.check()
        for b in range(30):
            last = path[b, kept[b] - 1]
            assert nxt[b] == best[c.cu[b] + last]


def test_nothing_left_and_odd_rows():
    """Draft and target equal but the token refused (a token of probability 0), rows of zeros, NaN and
    negative entries, random numbers at the ends."""
    c = Case([2] * 6, 40, True, 1, back=1)
    for b in range(6):
        t = 2 * b
        c.draft[t] = c.target[t]
        c.target[t, 7] = c.draft[t, 7] = 0.0
        c.tokens[t + 1] = 7                              # never stays: 0 < 0 is false; nothing is left
        c.uniforms[t] = [0.0, 0.3, 0.999, 0.5, 1 - 2.0 ** -24, 0.7][b]
    c.target[6] = c.draft[6] = 0.0                       # sequence 3: a row of zeros
    c.target[8, :20] = np.nan                            # sequence 4: the last token with a weight
    c.target[8, 30:] = -1.0
    c.check()
    c = Case([4, 4], 90, False, 2, back=1)
    c.tokens[[1, 5]] = [-1, 90]                          # no tokens: never kept
    c.tokens[6] = c.tokens[7]
    c.check()


def test_same_token_twice():
    """Siblings with one token: the second is judged by what the first one's refusal left."""
    for drawn in (True, False):
        c = Case([6] * 60, 12, drawn, 4, back=1)
        c.parents = np.tile(np.array([-1, 0, 0, 0, 0, 0], np.int32), 60)
        c.tokens = np.random.Generator(np.random.PCG64(1)).integers(0, 4, size=360).astype(np.int32)
        _, kept, _, _ = c.check()
        assert (kept == 1).any() and (kept == 2).any()


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("V", [300, 20011])
def test_many_children(V, drawn):
    """Hundreds of children of one node, nearly all refused (they lie in several 64s of nodes), and a
    chain behind the last one."""
    c = Case([330, 200], V, drawn, 17, back=1)
    for b, n in enumerate(c.n):
        t0 = c.cu[b]
        c.parents[t0 + 1:t0 + n] = 0
        c.parents[t0 + n - 2], c.parents[t0 + n - 1] = n - 3, n - 2
        if not drawn:
            order = np.argsort(c.target[t0])                 # the least likely tokens, each once
            c.tokens[t0 + 1:t0 + n] = np.resize(order[:max(64, V // 2)], n - 1)
    c.uniforms[:] = np.maximum(c.uniforms, 0.3)
    got = c.check()
    c.uniforms[[0, 330]] = [0.0, 1 - 2.0 ** -24]
    c.check()


@pytest.mark.parametrize("drawn", [True, False])
def test_distribution(drawn):
    """The first new token is distributed as the target's first row, whatever the draft: over N draws a
    token's count is within 5 sqrt(N p (1 - p)) + 1 of N p (a deviation of 5 sigma: below 1e-6 each)."""
    N, V = 20000, 8
    c = Case([4], V, drawn, 11, back=1, sharp=1.0, away=1.0)
    rng = np.random.Generator(np.random.PCG64(3))
    parents = np.tile(np.array([-1, 0, 0, 1], np.int32), N)
    target, q = np.tile(c.target, (N, 1)), _softmax(rng.standard_normal((4, V)))
    if drawn:
        cum = np.cumsum(q.astype(np.float64), 1)
        src = np.tile(np.array([0, 0, 0, 1]), N)
        tokens = (cum[src] < rng.random(4 * N)[:, None] * cum[src][:, -1:]).sum(1).clip(0, V - 1).astype(np.int32)
    else:
        tokens = np.tile(np.array([0, 3, 5, 2], np.int32), N)
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()      # noqa: E731
    path = torch.empty(N, 4, dtype=torch.int32, device="cuda")
    kept, nxt, ctx = (torch.empty(N, dtype=torch.int32, device="cuda") for _ in range(3))
    pcr.verify_drafts(_i32(4 * np.arange(N + 1)), cuda(parents), cuda(tokens), cuda(target),
                      cuda(np.tile(q, (N, 1))) if drawn else None, cuda(rng.random(4 * N).astype(np.float32).clip(0, 1 - 2.0 ** -24)),
                      _i32(np.zeros(N)), path, kept, nxt, ctx)
    path, kept, nxt = path.cpu().numpy(), kept.cpu().numpy(), nxt.cpu().numpy()
    first = np.where(kept > 1, tokens.reshape(N, 4)[np.arange(N), np.maximum(path[:, 1], 0)], nxt)
    p = c.target[0].astype(np.float64)
    p /= p.sum()
    count = np.bincount(first, minlength=V)
    assert (np.abs(count - N * p) <= 5 * np.sqrt(N * p * (1 - p)) + 1).all(), (count / N, p)


def test_graph_replays():
    c = Case([6, 3, 9, 1], 3001, True, 21, 3)
    B = c.B
    cuda = lambda a: torch.from_numpy(a).cuda()                  # noqa: E731
    ins = [_i32(c.cu), cuda(c.parents), cuda(c.tokens), cuda(c.target), cuda(c.draft), cuda(c.uniforms), _i32(c.p)]
    outs = [torch.zeros(B, c.cap, dtype=torch.int32, device="cuda")] + [torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(3)]
    ws = torch.empty(max(16, pcr.verify_drafts_workspace_bytes(B, c.T, c.V)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pcr.verify_drafts(*ins, *outs, workspace=ws)
    for k in range(4):
        d = Case([6, 3, 9, 1], 3001, True, 30 + k, 3)
        c.uniforms, c.target, c.draft, c.tokens = d.uniforms, d.target, d.draft, d.tokens
        for t, a in zip(ins[2:6], (c.tokens, c.target, c.draft, c.uniforms)):
            t.copy_(cuda(a))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, c.want()):
            assert np.array_equal(o.cpu().numpy(), w)
