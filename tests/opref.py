"""Plain references of the operators around the pool (block assignment and release, rotary
positions, cross attention), written from their definitions: whole numbers in Python, values
in 64 bits on the CPU. Test infrastructure only."""
import numpy as np
import torch

BS = 16
I32_MAX = 2 ** 31 - 1


def _blocks(n):
    return -(-n // BS)


def assign(p, s, bt, free, count, num_blocks, cap):
    """(block tables, slots, positions, cu, context lens, count out, status)."""
    bt = bt.copy()
    B, W = bt.shape
    count = min(max(int(count), 0), len(free))
    served, taken, tokens = 0, 0, 0
    slots, positions = np.full(cap, -1, np.int32), np.zeros(cap, np.int32)
    cu, ctx = np.zeros(B + 1, np.int32), np.array(p, np.int32)
    for b in range(B):
        pb, sb = int(p[b]), int(s[b])
        ok = served == b and pb >= 0 and sb >= 0
        if ok:
            held, need = _blocks(pb), _blocks(pb + sb)
            ok = need <= W and taken + need - held <= count and tokens + sb <= cap
        if ok:
            for e in range(held, need):
                bt[b, e] = free[count - 1 - taken]
                taken += 1
            for t in range(pb, pb + sb):
                blk = int(bt[b, t // BS])
                slots[tokens] = blk * BS + t % BS if 0 <= blk < num_blocks else -1
                positions[tokens] = t
                tokens += 1
            ctx[b] = pb + sb
            served += 1
        cu[b + 1] = tokens
    return bt, slots, positions, cu, ctx, count - taken, np.array([served, taken, tokens], np.int32)


def release(lens, keep, bt, free, count):
    """(free blocks, count out, status)."""
    free = free.copy()
    B, W = bt.shape
    count = min(max(int(count), 0), len(free))
    ids = []
    for b in range(B):
        first, last = _blocks(max(int(keep[b]), 0)), _blocks(min(int(lens[b]), W * BS))
        ids += [int(bt[b, e]) for e in range(first, last)]
    n = len(ids)
    if n > len(free) - count:
        return free, count, np.array([0, 0, min(n, I32_MAX)], np.int32)
    free[count:count + n] = ids[::-1]
    return free, count + n, np.array([B, n, n], np.int32)


def rotate(x, positions, inv_freq, axis, interleaved, scale=1.0, inverse=False):
    """x [T][H][d] (float64 tensor) rotated, and the size of what each result was formed from
    (|x1| + |x2| of its pair, 0 for dims passed through)."""
    half = len(inv_freq)
    y, size = x.clone(), torch.zeros_like(x)
    for j in range(half):
        i1, i2 = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        a = positions[int(axis[j])].double() * float(inv_freq[j])
        c, s = scale * torch.cos(a)[:, None], scale * torch.sin(a)[:, None]
        if inverse:
            s = -s
        y[:, :, i1] = x[:, :, i1] * c - x[:, :, i2] * s
        y[:, :, i2] = x[:, :, i2] * c + x[:, :, i1] * s
        size[:, :, i1] = size[:, :, i2] = x[:, :, i1].abs() + x[:, :, i2].abs()
    return y, size


def cross(q, pool_k, pool_v, bt, key_lens, cu, Hkv, sm_scale):
    """Cross attention in 64 bits, and sum_j w_j |v_j - out| per element (what the rounding of
    the weights can move). q [T][Hq][d]; the pools [blocks][Hkv][16*d], all float64."""
    T, Hq, d = q.shape
    G = Hq // Hkv
    out, dev = torch.zeros_like(q), torch.zeros_like(q)
    for b in range(len(key_lens)):
        n, t0, t1 = int(key_lens[b]), int(cu[b]), int(cu[b + 1])
        if n == 0 or t0 == t1:
            continue
        blocks = torch.as_tensor(np.asarray(bt[b][:_blocks(n)], np.int64))
        for h in range(Hq):
            k = pool_k[blocks, h // G].reshape(-1, d)[:n]
            v = pool_v[blocks, h // G].reshape(-1, d, BS).transpose(1, 2).reshape(-1, d)[:n]
            w = torch.softmax(q[t0:t1, h] @ k.t() * sm_scale, dim=1)
            out[t0:t1, h] = w @ v
            for a in range(t0, t1, 64):
                e = min(t1, a + 64)
                ww = w[a - t0:e - t0]
                dev[a:e, h] = torch.stack([(ww * (v[:, x][None] - out[a:e, h, x][:, None]).abs()).sum(1)
                                           for x in range(d)], dim=1)
    return out, dev
