"""GPU: block assignment and release against their definitions in Python, whole numbers all
equal: lengths of zero and one and far beyond a workgroup's sequences, every reason to refuse
a sequence, bad ids and counts, the arrays' ends, in-place updates and graph replays."""
import numpy as np
import pytest
import torch

import opref
from paper_2603_23049_amd import pcr

pytestmark = pytest.mark.gpu
BS = 16
GUARD = 12345


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


def _guarded(n):
    """n elements inside a longer array of guard values."""
    whole = torch.full((n + 64,), GUARD, dtype=torch.int32, device="cuda")
    return whole, whole[32:32 + n]


def _setup(p, s, num_blocks, seed, free_n=None, W=None):
    rng = np.random.Generator(np.random.PCG64(seed))
    perm = rng.permutation(num_blocks).astype(np.int32)
    held = [max(0, -(-int(x) // BS)) if x < 2 ** 28 else 0 for x in p]
    need = [max(1, -(-(int(a) + int(b)) // BS)) for a, b in zip(p, s)]
    W = W or min(max(need + [1]), 4096)
    bt = np.full((len(p), W), -1, np.int32)
    at = 0
    for b, h in enumerate(held):
        h = min(h, W)
        bt[b, :h] = perm[at:at + h]
        at += h
    free = perm[at:]
    if free_n is not None:
        free = free[:free_n]
    return bt, free


def _assign(p, s, bt, free, count, num_blocks, cap, with_positions=True):
    B = len(p)
    arrays = dict(slots=_guarded(cap), pos=_guarded(cap), cu=_guarded(B + 1), ctx=_guarded(B), cnt=_guarded(1),
                  status=_guarded(3), bt=_guarded(bt.size))
    btd = arrays["bt"][1].view(bt.shape)
    btd.copy_(_i32(bt))
    pcr.assign_blocks(_i32(p), _i32(s), btd, _i32(free), _i32([count]), num_blocks, arrays["slots"][1],
                      arrays["cu"][1], arrays["ctx"][1], arrays["cnt"][1], arrays["status"][1],
                      positions=arrays["pos"][1] if with_positions else None)
    torch.cuda.synchronize()
    for name, (whole, inner) in arrays.items():
        w = whole.cpu().numpy()
        assert (w[:32] == GUARD).all() and (w[32 + inner.numel():] == GUARD).all(), f"{name}: written outside"
    return btd.cpu().numpy(), *(arrays[k][1].cpu().numpy() for k in ("slots", "pos", "cu", "ctx", "cnt", "status"))


def _check(p, s, bt, free, count, num_blocks, cap):
    got = _assign(p, s, bt, free, count, num_blocks, cap)
    want = opref.assign(p, s, bt, free, count, num_blocks, cap)
    for name, g, w in zip(("tables", "slots", "positions", "cu", "ctx", "count", "status"), got, want):
        assert np.array_equal(g.reshape(-1), np.asarray(w, np.int32).reshape(-1)), name
    return want


@pytest.mark.parametrize("B,p_max,s_max,extra", [(1, 0, 1, 0), (1, 40, 1, 3), (3, 33, 0, 5), (64, 500, 1, 0), (64, 500, 1, 9),
                                           (65, 100, 90, 0), (700, 50, 40, 1000), (1025, 40, 3, 0), (2300, 20, 30, 17),
                                           (5, 3000, 9000, 0), (1, 17, 20000, 4000), (255, 64, 200, 1), (1024, 0, 33, 2)])
def test_assign_equals_definition(B, p_max, s_max, extra):
    rng = np.random.Generator(np.random.PCG64(B * 7 + s_max))
    p = rng.integers(0, p_max + 1, size=B)
    s = rng.integers(min(1, s_max) if B == 64 else 0, s_max + 1, size=B)
    num_blocks = int(sum(-(-(a + b) // BS) for a, b in zip(p, s))) + 5
    bt, free = _setup(p, s, num_blocks, B)
    want = _check(p, s, bt, free, len(free), num_blocks, int(s.sum()) + extra)
    assert want[-1][0] == B
    got = _assign(p, s, bt, free, len(free), num_blocks, int(s.sum()) + extra, with_positions=False)
    assert np.array_equal(got[1], want[1]) and (got[2] == GUARD).all()


def test_many_sequences():
    """Tiles of several rows per thread (they grow with the sequences), for both directions."""
    B = 40000
    rng = np.random.Generator(np.random.PCG64(17))
    p, s = rng.integers(0, 40, size=B), rng.integers(0, 3, size=B)
    num_blocks = int(sum(-(-(a + b) // BS) for a, b in zip(p, s))) + 5
    bt, free = _setup(p, s, num_blocks, 6)
    table = _check(p, s, bt, free, len(free), num_blocks, int(s.sum()) + 700)[0].reshape(B, -1)
    lens, keep = p + s, np.where(rng.random(B) < 0.5, p, 0)
    stack = _i32(np.full(num_blocks, -9))
    count, status = _i32([3]), _i32([0, 0, 0])
    pcr.release_blocks(_i32(lens), _i32(keep), _i32(table), stack, count, num_blocks, count, status)
    want = [table[b, e] for b in range(B) for e in range(-(-keep[b] // BS), -(-lens[b] // BS))]
    assert status.tolist() == [B, len(want), len(want)] and count.item() == 3 + len(want)
    got = stack.cpu().numpy()
    assert np.array_equal(got[3:3 + len(want)], np.array(want[::-1])) and (got[3 + len(want):] == -9).all()


def test_assign_at_block_edges():
    p = [0, 15, 16, 17, 31, 32, 0, 16, 0]
    s = [16, 1, 1, 15, 2, 16, 17, 0, 0]
    bt, free = _setup(p, s, 40, 3)
    _check(p, s, bt, free, len(free), 40, sum(s))


@pytest.mark.parametrize("why", ["negative_p", "negative_s", "row", "blocks", "slots", "huge", "first", "none_left",
                                 "count_above", "count_below", "count_part"])
@pytest.mark.parametrize("B,at", [(6, 3), (1500, 1200), (1500, 1024)])
def test_assign_refuses_from_the_first_that_does_not_fit(why, B, at):
    rng = np.random.Generator(np.random.PCG64(B + at))
    p, s = rng.integers(0, 40, size=B), rng.integers(1, 20, size=B)
    num_blocks = int(sum(-(-(a + b) // BS) for a, b in zip(p, s))) + 3
    bt, free = _setup(p, s, num_blocks, 5, W=8)
    count, cap = len(free), int(s.sum()) + 2
    if why == "negative_p":
        p[at] = -1
    elif why == "negative_s":
        s[at] = -5
    elif why == "row":
        s[at] = 8 * BS + 1
    elif why == "blocks":
        count = int(sum(-(-(a + b) // BS) - -(-a // BS) for a, b in zip(p[:at + 1], s[:at + 1])))
        s[at] += BS
    elif why == "slots":
        cap = int(s[:at + 1].sum()) - 1
    elif why == "huge":
        p[at], s[at] = 2 ** 31 - 1, 2 ** 31 - 1
        s[at + 1] = 2 ** 31 - 1
    elif why == "first":
        p[0] = -2 ** 31
    elif why == "none_left":
        count = 0
    elif why == "count_above":
        count = 2 ** 31 - 1
    elif why == "count_below":
        count = -7
    elif why == "count_part":
        count = len(free) // 2
    _check(p, s, bt, free, count, num_blocks, cap)


def test_assign_bad_ids_get_no_slot():
    p, s = [20, 5, 0], [20, 3, 40]
    bt, free = _setup(p, s, 30, 7)
    bt[0, 1] = -3
    bt[1, 0] = 30
    free = free.copy()
    free[-2] = 2 ** 31 - 1
    _check(p, s, bt, free, len(free), 30, 70)


def test_assign_empty_batch_marks_the_rows():
    bt, free = np.zeros((0, 4), np.int32), np.arange(3, dtype=np.int32)
    _check([], [], bt, free, 3, 8, 50)
    _check([], [], bt, np.zeros(0, np.int32), 0, 8, 5000)


@pytest.mark.parametrize("B,len_max,extra", [(1, 1, 0), (1, 5000, 0), (7, 100, 3), (300, 700, 0), (1024, 40, 1), (1700, 90, 0),
                                             (3, 40000, 9)])
def test_release_equals_definition(B, len_max, extra):
    rng = np.random.Generator(np.random.PCG64(B))
    lens = rng.integers(0, len_max + 1, size=B)
    keep = np.maximum(lens - rng.integers(-3, len_max + 2, size=B), -4)
    lens[-1], keep[-1] = len_max, 0
    num_blocks = int(sum(-(-int(x) // BS) for x in lens)) + 4
    bt, rest = _setup(lens, np.zeros(B, int), num_blocks, B)
    n = int(opref.release(lens, keep, bt, np.zeros(1 << 20, np.int32), 0)[1])
    for cap in (n + 4 + extra, n + 3, n + 2):         # room, just room, one short (4 free ids at the start, or 3)
        count = min(len(rest), 3)
        whole, free = _guarded(cap)
        f0 = np.full(cap, -7, np.int32)
        f0[:count] = rest[:count]
        free.copy_(_i32(f0))
        cnt, status = _guarded(1), _guarded(3)
        pcr.release_blocks(_i32(lens), _i32(keep), _i32(bt), free, _i32([count]), num_blocks, cnt[1], status[1])
        torch.cuda.synchronize()
        wf, wc, ws = opref.release(lens, keep, bt, f0, count)
        assert np.array_equal(free.cpu().numpy(), wf) and int(cnt[1]) == wc
        assert np.array_equal(status[1].cpu().numpy(), ws)
        w = whole.cpu().numpy()
        assert (w[:32] == GUARD).all() and (w[32 + cap:] == GUARD).all()


def test_release_bad_lengths_and_counts():
    bt = np.arange(12, dtype=np.int32).reshape(3, 4)
    for lens, keep, count in (([-5, 1000, 2 ** 31 - 1], [0, 3, -2 ** 31], 0), ([64, 64, 64], [64, 65, 2 ** 31 - 1], 2),
                              ([64, 0, 1], [0, 0, 0], -9), ([64, 0, 1], [0, 0, 0], 2 ** 31 - 1)):
        free = np.arange(100, 130, dtype=np.int32)
        fd, cnt, status = _i32(free), _i32([0]), _i32([0, 0, 0])
        pcr.release_blocks(_i32(lens), _i32(keep), _i32(bt), fd, _i32([count]), 40, cnt, status)
        wf, wc, ws = opref.release(lens, keep, bt, free, count)
        assert np.array_equal(fd.cpu().numpy(), wf) and int(cnt) == wc and np.array_equal(status.cpu().numpy(), ws)


def test_release_undoes_assign_in_place():
    rng = np.random.Generator(np.random.PCG64(11))
    p, s = rng.integers(0, 90, size=130), rng.integers(0, 70, size=130)
    num_blocks = int(sum(-(-(a + b) // BS) for a, b in zip(p, s))) + 9
    bt, free = _setup(p, s, num_blocks, 2)
    pd, sd, btd, fd, cnt = _i32(p), _i32(s), _i32(bt), _i32(free), _i32([len(free)])
    slots, cu, status = _i32(np.zeros(int(s.sum()))), _i32(np.zeros(131)), _i32([0, 0, 0])
    pcr.assign_blocks(pd, sd, btd, fd, cnt, num_blocks, slots, cu, pd, cnt, status)     # lengths and count in place
    assert np.array_equal(pd.cpu().numpy(), p + s)
    left = int(cnt)
    fd[left:] = -1
    pcr.release_blocks(pd, _i32(p), btd, fd, cnt, num_blocks, cnt, status)
    assert int(cnt) == len(free) and np.array_equal(fd.cpu().numpy(), free)


@pytest.mark.parametrize("B", [3, 200])
def test_graph_replays_are_consecutive_decode_steps(B):
    """One captured step, lengths and count updated in place: each replay is the next token of
    every sequence, beside eager work and synchronisations."""
    steps, cap = 40, B + 2
    p0 = np.random.Generator(np.random.PCG64(B)).integers(0, 50, size=B).astype(np.int32)
    num_blocks = int(sum(-(-(int(a) + steps) // BS) for a in p0)) + 2
    bt, free = _setup(p0, np.full(B, steps), num_blocks, 4)
    state = [_i32(p0), _i32(bt), _i32([len(free)])]
    sd, fd = _i32(np.ones(B)), _i32(free)
    slots, pos, cu, status = (_i32(np.zeros(n)) for n in (cap, cap, B + 1, 3))

    def step():
        pcr.assign_blocks(state[0], sd, state[1], fd, state[2], num_blocks, slots, cu, state[0], state[2], status,
                          positions=pos)

    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        step()
    torch.cuda.synchronize()
    p, t, count = p0.copy(), bt, len(free)
    for i in range(steps):
        if i % 7 == 3:
            step()                         # an eager step in between
        else:
            g.replay()
        t, wslots, wpos, wcu, p, count, wstatus = opref.assign(p, np.ones(B, int), t, free, count, num_blocks, cap)
        torch.cuda.synchronize()
        assert np.array_equal(slots.cpu().numpy(), wslots) and np.array_equal(pos.cpu().numpy(), wpos), i
        assert np.array_equal(state[0].cpu().numpy(), p) and int(state[2]) == count, i
        assert np.array_equal(state[1].cpu().numpy(), t) and np.array_equal(status.cpu().numpy(), wstatus), i
        _ = torch.zeros(1000, device="cuda").sum().item()


def test_on_another_stream():
    p, s = [30, 5], [9, 40]
    bt, free = _setup(p, s, 30, 1)
    st = torch.cuda.Stream()
    args = [_i32(p), _i32(s), _i32(bt), _i32(free), _i32([len(free)])]
    slots, cu, ctx, cnt, status = (_i32(np.zeros(n)) for n in (60, 3, 2, 1, 3))
    torch.cuda.synchronize()
    pcr.assign_blocks(*args, 30, slots, cu, ctx, cnt, status, stream=st)
    st.synchronize()
    want = opref.assign(p, s, bt, free, len(free), 30, 60)
    assert np.array_equal(slots.cpu().numpy(), want[1]) and np.array_equal(ctx.cpu().numpy(), want[4])
