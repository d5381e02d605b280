"""Plain references of the operators of a speculative step (draft trees, tree attention,
verification, compaction), written from their definitions: whole numbers in Python, values in
64 bits on the CPU. Test infrastructure only."""
import numpy as np
import torch

BS = 16


def random_parents(rng, n, back=6):
    """A tree of n nodes: node 0 follows the cached tokens, every other one a node before it."""
    return [-1] + [max(0, i - 1 - int(rng.integers(0, back))) for i in range(1, n)] if n else []


def draft_tree(cu, parents, p, T, words, visible, positions):
    """(visible as uint64 [T][words], positions [T]); rows behind the last sequence as given."""
    visible, positions = visible.copy(), positions.copy()
    for b in range(len(p)):
        t0, n = int(cu[b]), int(cu[b + 1]) - int(cu[b])
        way = []                                   # of every node: itself and its ancestors, or None
        for i in range(n):
            par = int(parents[t0 + i])
            if i >= 64 * words or not -1 <= par < i:
                way.append(None)
            elif par < 0:
                way.append([i])
            else:
                way.append(None if way[par] is None else way[par] + [i])
        for i in range(n):
            bits = [0] * words
            for k in way[i] or []:
                bits[k // 64] |= 1 << (k % 64)
            visible[t0 + i] = np.array(bits, np.uint64)
            positions[t0 + i] = int(p[b]) + (len(way[i]) - 1 if way[i] else 0)
    return visible, positions


def words_of(cu, parents, words):
    T = len(parents)
    B = len(cu) - 1
    return draft_tree(cu, parents, np.zeros(B, np.int32), T, words, np.zeros((T, words), np.uint64),
                      np.zeros(T, np.int32))[0]


def tree_attn(q, pool_k, pool_v, bt, p, cu, visible, Hkv, sm_scale):
    """Tree attention in 64 bits, and sum_j w_j |v_j - out| per element (what the rounding of the
    weights can move). q [T][Hq][d]; the pools [blocks][Hkv][16*d], all float64; visible uint64."""
    T, Hq, d = q.shape
    G = Hq // Hkv
    out, dev = torch.zeros_like(q), torch.zeros_like(q)
    for b in range(len(p)):
        t0, n = int(cu[b]), int(cu[b + 1]) - int(cu[b])
        for i in range(n):
            seen = list(range(int(p[b])))
            seen += [int(p[b]) + k for k in range(n) if int(visible[t0 + i][k // 64]) >> (k % 64) & 1]
            if not seen:
                continue
            pos = np.array(seen)
            blk = torch.as_tensor(np.asarray(bt[b], np.int64)[pos // BS])
            off = torch.as_tensor(pos % BS)
            for g in range(Hkv):
                k = pool_k.view(-1, Hkv, BS, d)[blk, g, off]
                v = pool_v.view(-1, Hkv, d, BS)[blk, g, :, off]
                qq = q[t0 + i, g * G:(g + 1) * G]
                w = torch.softmax(qq @ k.t() * sm_scale, dim=1)
                o = w @ v
                out[t0 + i, g * G:(g + 1) * G] = o
                dev[t0 + i, g * G:(g + 1) * G] = (w[:, :, None] * (v[None] - o[:, None]).abs()).sum(1)
    return out, dev


def verify(cu, parents, tokens, target, draft, uniforms, p, path_cap):
    """(path, accepted_lens, next_tokens, context_lens); probabilities as float32 arrays."""
    B = len(p)
    path = np.full((B, path_cap), -1, np.int32)
    kept, nxt = np.zeros(B, np.int32), np.full(B, -1, np.int32)
    clean = lambda r: np.where(r > 0, r, 0.0)       # noqa: E731  (NaN and negative values count as 0)
    with np.errstate(invalid="ignore"):
        for b in range(B):
            t0, n = int(cu[b]), int(cu[b + 1]) - int(cu[b])
            if n == 0:
                continue
            V = target.shape[1]
            way, u, a, Z, gone = [0], 0, 0.0, 1.0, set()

            def rest():
                P = target[t0 + u].astype(np.float64)
                if draft is None:
                    r = clean(P)
                    r[list(gone)] = 0.0
                    return r
                return clean(P - a * draft[t0 + u].astype(np.float64))

            for i in range(1, n):
                if len(way) >= path_cap:
                    break
                x = int(tokens[t0 + i])
                if int(parents[t0 + i]) != u or not 0 <= x < V:
                    continue
                w = float(rest()[x])
                ask = float(uniforms[t0 + i]) * (float(draft[t0 + u, x]) if draft is not None else 1.0) * Z
                if ask < w:
                    u, a, Z, gone = i, 0.0, 1.0, set()
                    way.append(i)
                elif draft is not None:
                    a = a + Z
                    Z = float(rest().sum())
                else:
                    Z -= w
                    gone.add(x)
            r = rest()
            if not r.sum() > 0:
                r = clean(target[t0 + u].astype(np.float64))
            over = np.nonzero(np.cumsum(r) > float(uniforms[t0]) * r.sum())[0]
            some = np.nonzero(r > 0)[0]
            last = int(some[-1]) if len(some) else 0
            nxt[b] = min(int(over[0]), last) if len(over) else last
            path[b, :len(way)] = way
            kept[b] = len(way)
    return path, kept, nxt, np.asarray(p, np.int32) + kept


def compact(k, v, bt, p, path, kept):
    """(K, V) of one layer, as arrays [blocks][Hkv][16*d] of 16-bit patterns."""
    nb, Hkv, n = k.shape
    d = n // BS
    k, v = k.copy(), v.copy()
    k0, v0 = k.copy().reshape(nb, Hkv, BS, d), v.copy().reshape(nb, Hkv, d, BS)
    kk, vv = k.reshape(nb, Hkv, BS, d), v.reshape(nb, Hkv, d, BS)
    W = bt.shape[1]
    for b in range(len(p)):
        before = -1
        for i in range(min(int(kept[b]), path.shape[1])):
            x, pb = int(path[b, i]), int(p[b])
            if pb < 0 or x <= before:
                break
            before = x
            if x == i:
                continue
            s, t = pb + x, pb + i
            if s >= W * BS or not (0 <= bt[b, s // BS] < nb and 0 <= bt[b, t // BS] < nb):
                break
            kk[bt[b, t // BS], :, t % BS] = k0[bt[b, s // BS], :, s % BS]
            vv[bt[b, t // BS], :, :, t % BS] = v0[bt[b, s // BS], :, :, s % BS]
    return k, v
