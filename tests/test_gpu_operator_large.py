"""GPU: the operators around the pool where offsets pass 32 bits (a pool of 2^32 elements, rows
far apart) and where two calls run at once. The same contents in a small pool, or the same call
alone, give the bits to compare with; those cases are held to 64-bit definitions elsewhere."""
import numpy as np
import pytest
import torch

from paper_2603_23049_amd import pcr

pytestmark = pytest.mark.gpu
BS = 16


def _bf16(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)


def _i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def _rope(d, axes=1):
    f = (10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)
    return pcr.Rope(f, np.arange(d // 2) % axes, axes)


@pytest.mark.parametrize("T", [20, 3000])                  # rows of single waves, tiles
def test_pool_beyond_32_bit_offsets(T):
    gen = torch.Generator(device="cuda").manual_seed(T)
    Hq, Hkv, d = 16, 16, 128
    nb, small = (1 << 32) // (Hkv * BS * d) + 400, 400     # K and V: 2^32 elements and 400 blocks each
    n = -(-T // BS)
    far = torch.randperm(300, generator=gen, device="cuda")[:n] + (nb - 300)
    far[::3] = torch.arange(0, n, 3, device="cuda")        # every third block at the pool's start
    near = torch.arange(n, device="cuda") + 5
    pools, outs, res = [], [], []
    q, k, v = _bf16(gen, T, Hq, d), _bf16(gen, T, Hkv, d), _bf16(gen, T, Hkv, d)
    pos = torch.randint(0, 10 ** 6, (1, T), generator=gen, device="cuda", dtype=torch.int32)
    off = torch.arange(T, device="cuda") % BS
    for blocks, size in ((far, nb), (near, small)):
        pool = pcr.KVPool(torch.empty(size, Hkv, BS * d, dtype=torch.bfloat16, device="cuda"),
                          torch.empty(size, Hkv, BS * d, dtype=torch.bfloat16, device="cuda"), Hkv, d)
        slots = (blocks.repeat_interleave(BS)[:T] * BS + off).to(torch.int32)
        out = torch.empty_like(q)
        pcr.rope_append_kv(_rope(d), pool, q, k, v, pos, slots, Hq, out)
        outs.append(out)
        rows = torch.arange(T, device="cuda")
        pools.append((pool.k[blocks].view(n, Hkv, BS, d)[rows // BS, :, off], pool.v[blocks].view(n, Hkv, d, BS)[rows // BS, :, :, off]))
        table = blocks.to(torch.int32)[None].contiguous()
        for s in (1, 40):                                  # few rows, row tiles
            got = torch.empty(s, Hq, d, dtype=torch.bfloat16, device="cuda")
            cu = np.array([0, s], np.int32)
            pcr.cross_attn(out[:s] if s <= T else out.repeat(2, 1, 1)[:s], pool, table, _i32([T]), _i32(cu), [T], cu, Hq, got)
            res.append(got)
        del pool
    assert torch.equal(outs[0], outs[1])
    assert torch.equal(pools[0][0], pools[1][0]) and torch.equal(pools[0][1], pools[1][1])
    assert torch.equal(pools[1][1], v)
    assert torch.equal(res[0], res[2]) and torch.equal(res[1], res[3]) and torch.isfinite(res[1].float()).all()


def test_rows_far_apart():
    gen = torch.Generator(device="cuda").manual_seed(3)
    T, H, d, stride = 6, 2, 64, (1 << 29) + 8              # the last row starts past 2^31 elements
    wide = torch.empty(stride * (T - 1) + H * d, dtype=torch.bfloat16, device="cuda")
    x = _bf16(gen, T, H, d)
    view = wide.as_strided((T, H, d), (stride, d, 1))
    view.copy_(x)
    pos = torch.randint(0, 5000, (2, T), generator=gen, device="cuda", dtype=torch.int32)
    want = torch.empty_like(x)
    pcr.rope_rows(_rope(d, 2), x, pos, want)
    pcr.rope_rows(_rope(d, 2), view, pos, view)
    assert torch.equal(view, want)


def test_two_calls_at_once():
    """Calls on two streams, each with a workspace of its own, eager and as two graphs replayed together."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    Hq, Hkv, d = 8, 2, 128
    pool = pcr.KVPool(_bf16(gen, 900, Hkv, BS * d), _bf16(gen, 900, Hkv, BS * d), Hkv, d)
    calls = []
    for keys, rows in (([9000, 300, 4000], [1, 2, 1]), ([5000, 0, 2000], [30, 2, 1])):
        n, cu = np.array(keys, np.int32), np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        bt = torch.randint(0, 900, (3, 563), generator=gen, device="cuda", dtype=torch.int32)
        q = _bf16(gen, int(cu[-1]), Hq, d)
        size = pcr.cross_attn_workspace_bytes(3, int(cu[-1]), Hq, Hkv, d, max(keys))
        calls.append((q, pool, bt, _i32(n), _i32(cu), n, cu, Hq, torch.empty_like(q), torch.empty(size, dtype=torch.uint8, device="cuda")))
    want = []
    for *a, out, ws in calls:
        pcr.cross_attn(*a, out, workspace=ws)
        want.append(out.clone())
    streams = [torch.cuda.Stream() for _ in calls]
    graphs = [torch.cuda.CUDAGraph() for _ in calls]
    torch.cuda.synchronize()
    for g, (*a, out, ws) in zip(graphs, calls):
        with torch.cuda.graph(g):
            pcr.cross_attn(*a, out, workspace=ws)
    for replay in (False, True):
        for *a, out, ws in calls:
            out.fill_(float("nan"))
        torch.cuda.synchronize()
        for _ in range(20):
            for s, g, (*a, out, ws) in zip(streams, graphs, calls):
                with torch.cuda.stream(s):
                    if replay:
                        g.replay()
                    else:
                        pcr.cross_attn(*a, out, workspace=ws)
        torch.cuda.synchronize()
        for w, c in zip(want, calls):
            assert torch.equal(c[-2], w)
