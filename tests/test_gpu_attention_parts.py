"""GPU: ragged batches on 1, 2 and 4 kv heads, whose row tiles are dealt in parts to the XCDs that share a
head: each sequence's rows are those of a launch of its own, bit for bit, whatever else is in the batch."""
import numpy as np
import pytest
import torch

from gpuio import attn_schedule, say
from paper_2603_23049_amd import pcr

pytestmark = pytest.mark.gpu
BS = 16


def _batch(p, s, Hq, Hkv, d, seed):
    need = [-(-(a + b) // BS) for a, b in zip(p, s)]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    k, v = (torch.randn(sum(need) + 1, Hkv, BS * d, device="cuda", generator=gen).bfloat16() for _ in range(2))
    bt = np.full((len(p), max(need)), -1, np.int32)
    perm = np.random.Generator(np.random.PCG64(seed)).permutation(sum(need) + 1).astype(np.int32)
    off = 0
    for b, n in enumerate(need):
        bt[b, :n] = perm[off:off + n]
        off += n
    q = torch.randn(sum(s), Hq, d, device="cuda", generator=gen).bfloat16()
    return q, pcr.KVPool(k, v, Hkv, d), torch.from_numpy(bt).cuda()


def _run(kind, q, pool, bt, p, s, Hq):
    cu = np.concatenate([[0], np.cumsum(s)]).astype(np.int32)
    lens = np.asarray(p if kind != "cross" else [a + b for a, b in zip(p, s)], np.int32)
    lens_d, cu_d = torch.from_numpy(lens).cuda(), torch.from_numpy(cu).cuda()
    out = torch.full_like(q, float("nan"))
    if kind == "causal":
        pcr.prefix_prefill_attn(q, pool, bt, lens_d, cu_d, lens, cu, Hq, out)
    elif kind == "cross":
        pcr.cross_attn(q, pool, bt, lens_d, cu_d, lens, cu, Hq, out)
    else:                                                   # each node sees the one before it and itself
        T, words = int(cu[-1]), -(-max(s) // 64)
        vis = np.zeros((T, words), np.uint64)
        for b, n in enumerate(s):
            for i in range(n):
                for j in (i - 1, i):
                    if j >= 0:
                        vis[cu[b] + i, j // 64] |= np.uint64(1 << (j % 64))
        pcr.tree_attn(q, pool, bt, lens_d, cu_d, lens, cu, torch.from_numpy(vis.view(np.int64)).cuda(), Hq, out)
    torch.cuda.synchronize()
    return out


def _draw(n, lo, hi, seed):
    return np.random.Generator(np.random.PCG64(seed)).integers(lo, hi + 1, size=n).tolist()


# prefix and new tokens of each sequence, Hq, Hkv, d
RAGGED = [
    (_draw(9, 0, 900, 1), _draw(9, 60, 300, 2), 8, 1, 128),         # one sequence more than parts
    (_draw(40, 0, 700, 3), _draw(40, 30, 200, 4), 4, 1, 64),
    (_draw(30, 0, 900, 5), _draw(30, 40, 150, 6), 14, 2, 128),
    (_draw(3, 0, 900, 7), [61, 200, 5], 28, 4, 128),
    (_draw(37, 0, 600, 8), _draw(37, 9, 61, 9), 28, 4, 128),
    ([700] * 20 + [100], [40] * 20 + [640], 16, 4, 64),             # the shortest text has the most rows
    (_draw(150, 0, 300, 10), _draw(150, 20, 60, 11), 8, 2, 64),     # two launches
    (_draw(30, 100, 900, 12) + [50], [40] * 30 + [1], 32, 4, 128),  # few decode rows among the row tiles
    (_draw(30, 100, 900, 13), [1] * 25 + [100] * 5, 8, 1, 128),     # many
]


@pytest.mark.parametrize("schedule", ["key_halves", "row_halves"])
@pytest.mark.parametrize("kind", ["causal", "cross", "tree"])
@pytest.mark.parametrize("case", range(len(RAGGED)))
def test_rows_are_those_of_a_launch_of_their_own(case, kind, schedule):
    p, s, Hq, Hkv, d = RAGGED[case]
    say(f"[gpu] parts case {case} {kind} {schedule}")
    q, pool, bt = _batch(p, s, Hq, Hkv, d, seed=case)
    cu = np.concatenate([[0], np.cumsum(s)])
    with attn_schedule(schedule):
        out = _run(kind, q, pool, bt, p, s, Hq)
        assert torch.isfinite(out).all()
        for b in range(0, len(p), max(1, len(p) // 12)):
            if kind != "causal" and s[b] * Hq // Hkv <= 32:
                continue                                    # alone it runs on the kernels of few rows
            alone = _run(kind, q[cu[b]:cu[b + 1]].clone(), pool, bt[b:b + 1], p[b:b + 1], s[b:b + 1], Hq)
            assert torch.equal(out[cu[b]:cu[b + 1]], alone), b


@pytest.mark.parametrize("kind", ["causal", "cross", "tree"])
@pytest.mark.parametrize("Hq,Hkv,n", [(8, 1, 9), (16, 2, 5), (28, 4, 3)])
def test_keys_cut_into_chunks(kind, Hq, Hkv, n):
    """The default schedule cuts these keys. Both results are weighted means of V with weights that are off by 2^-8
    of themselves at most, and so by 2^-7 max |v| each, and rounded to bf16 (2^-8 max |v|)."""
    p, s = _draw(n, 3000, 8000, Hkv), [16] * n
    say(f"[gpu] parts cut {kind} {Hq}/{Hkv}")
    q, pool, bt = _batch(p, s, Hq, Hkv, 128, seed=90 + Hkv)
    got = _run(kind, q, pool, bt, p, s, Hq)
    with attn_schedule("key_halves"):
        whole = _run(kind, q, pool, bt, p, s, Hq)
    assert not torch.equal(got, whole)                      # (the cut was made)
    bound = 2 * (2.0 ** -7 + 2.0 ** -8) * float(pool.v.float().abs().max())
    assert float((got.float() - whole.float()).abs().max()) <= bound
