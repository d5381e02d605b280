"""Measured cases of the operators of a speculative step over the paged KV cache: positions
and visible sets of a tree of drafted tokens (`tree`), attention of the tree's rows over the
cached tokens and their own ancestors (`attn`), the choice of the drafted tokens that stay, from
the target's probabilities and given random numbers (`verify`), and the move of their K/V
into consecutive slots in every layer (`compact`).

A sequence's nodes are rows cu[b] .. cu[b+1]-1. Node 0 is the last token of the text, the others
are drafted; parents[i] is the node that i follows (-1: the cached tokens).

`listed()` names the fixed cases and `draw()` makes more of the same ranges. With `own`
false, `run` computes the operators in plain torch operations; with `own` true it makes the
library's calls. Every tensor is made from the seed alone; lengths follow from the case.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BS = 16          # tokens per pool block
DEV = "cuda"


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # A decode step of 64 sequences with 16 nodes each: latency is all there is.
        dict(name="tree_64", kind="tree", B=64, n=16, n_min=16, words=1, back=6, lens=1),
        # 500 sequences with deep trees of up to 256 nodes.
        dict(name="tree_deep_500", kind="tree", B=500, n=256, n_min=100, words=4, back=2, lens=2),
        # One sequence, 8 nodes over 1000 cached tokens, a small model's heads: latency.
        dict(name="attn_one", kind="attn", B=1, Hq=8, Hkv=8, D=64, n=8, n_min=8, p=1000, p_min=1000, words=1, back=4,
             lens=3),
        # A decode step of 64 sequences with 16 nodes each (the 8B model's heads): reading K and V
        # is all there is.
        dict(name="attn_decode_64", kind="attn", B=64, Hq=32, Hkv=8, D=128, n=16, n_min=16, p=4352, p_min=2100, words=1,
             back=6, lens=4),
        # 37 ragged sequences, some without a prefix, trees of odd sizes, seven query heads per kv head.
        dict(name="attn_ragged_37", kind="attn", B=37, Hq=28, Hkv=4, D=128, n=61, n_min=1, p=1901, p_min=0, words=1,
             back=9, lens=5),
        # Full trees of 64 nodes on long texts with the 70B model's heads: matrix products.
        dict(name="attn_70b_32", kind="attn", B=32, Hq=64, Hkv=8, D=128, n=64, n_min=64, p=8000, p_min=7000, words=1,
             back=8, lens=6),
        # One chain of 5 drafted tokens: latency.
        dict(name="verify_one", kind="verify", B=1, n=6, n_min=6, V=32001, back=1, drawn=1, lens=7),
        # 64 sequences, chains of 4 drafted tokens with their probabilities: ordinary speculative
        # sampling.
        dict(name="verify_chain_64", kind="verify", B=64, n=5, n_min=5, V=128000, back=1, drawn=1, lens=8),
        # 48 trees of up to 24 drafted tokens that a draft proposed for certain (its best ones).
        dict(name="verify_best_48", kind="verify", B=48, n=25, n_min=9, V=50001, back=6, drawn=0, lens=9),
        # 128 trees of 12 drafted tokens drawn from the draft's probabilities, siblings from one row.
        dict(name="verify_tree_128", kind="verify", B=128, n=13, n_min=13, V=128000, back=4, drawn=1, lens=10),
        # 4 sequences that keep up to 4 of 8 nodes, the 8B model's 32 layers.
        dict(name="compact_4", kind="compact", B=4, Hkv=8, D=128, L=32, n=8, n_min=8, keep=4, lens=11),
        # 64 sequences that keep up to 8 of 32 nodes in the 70B model's 80 layers.
        dict(name="compact_64", kind="compact", B=64, Hkv=8, D=128, L=80, n=32, n_min=9, keep=8, lens=12),
    ]


HEADS = [(8, 8, 64), (32, 8, 128), (32, 8, 128), (64, 8, 128), (8, 1, 128), (16, 2, 128), (16, 4, 64), (28, 4, 128)]
MAX_FLOPS = 5.0e11      # a drawn case costs no more than the largest listed one
MAX_KEYS = 250000000    # elements of K
MAX_ROWS = 200000000    # probabilities


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    kind = rng.choice(["tree", "attn", "attn", "attn", "attn", "verify", "verify", "verify", "compact", "compact"])
    c = dict(kind=kind, lens=rng.randrange(1, 1 << 30))
    if kind == "tree":
        c["B"] = _log(rng, 1, 500)
        c["n"] = _log(rng, 1, 256)
        c["n_min"] = rng.choice([0, 1, c["n"]])
        c["words"] = (c["n"] + 63) // 64
        c["back"] = rng.choice([1, 2, 6, 20])
    elif kind == "attn":
        c["Hq"], c["Hkv"], c["D"] = rng.choice(HEADS)
        c["B"] = _log(rng, 1, 64)
        c["n"] = rng.choice([rng.randrange(1, 9), rng.randrange(4, 33), rng.randrange(16, 65), rng.randrange(65, 150)])
        c["n_min"] = rng.choice([0, 1, c["n"], c["n"]])
        c["p"] = _log(rng, 1, 16000)
        while (c["B"] * c["Hkv"] * c["D"] * c["p"] > MAX_KEYS
               or 4 * c["D"] * c["Hq"] * c["B"] * c["n"] * (c["p"] + c["n"]) > MAX_FLOPS):
            c["p"] = max(1, c["p"] * 2 // 3)
            c["B"] = max(1, c["B"] * 5 // 6)
        c["p_min"] = rng.choice([c["p"], c["p"] // 2, 0])
        c["words"] = (c["n"] + 63) // 64
        c["back"] = rng.choice([1, 3, 6, 20])
    elif kind == "verify":
        c["V"] = _log(rng, 1000, 200000)
        c["B"] = _log(rng, 1, 128)
        c["n"] = rng.choice([rng.randrange(1, 8), rng.randrange(5, 26), rng.randrange(5, 65)])
        while c["B"] * c["n"] * c["V"] > MAX_ROWS:
            c["B"] = max(1, c["B"] * 2 // 3)
            c["n"] = max(1, c["n"] * 5 // 6)
        c["n_min"] = rng.choice([1, c["n"], c["n"]])
        c["back"] = rng.choice([1, 1, 4, 8])
        c["drawn"] = rng.choice([0, 1, 1])
    else:
        _, c["Hkv"], c["D"] = rng.choice(HEADS)
        c["L"] = rng.choice([1, 16, 28, 32, 32, 80])
        c["B"] = _log(rng, 1, 64)
        c["n"] = rng.randrange(4, 65)
        c["n_min"] = rng.choice([1, c["n"]])
        c["keep"] = rng.randrange(2, min(c["n"], 9))
        while c["B"] * c["L"] * c["Hkv"] * c["D"] > 64 * 80 * 8 * 64:
            c["B"] = max(1, c["B"] * 2 // 3)
            c["L"] = max(1, c["L"] * 2 // 3)
    return c


def _spread(rng, lo, hi, n):
    """n whole numbers of [lo, hi], the largest among them."""
    v = rng.integers(lo, hi + 1, size=n)
    v[int(rng.integers(n))] = hi
    return v.astype(np.int32)


def _lens(c):
    """The case's cached tokens and nodes per sequence; with `compact` the paths that stay, too."""
    rng = np.random.Generator(np.random.PCG64(c["lens"]))
    n = _spread(rng, c["n_min"], c["n"], c["B"])
    if c["kind"] == "compact":
        # The tokens before the step's, as far as they share a block with them.
        p = rng.integers(0, BS, size=c["B"]).astype(np.int32)
        kept = np.minimum(_spread(rng, 1, c["keep"], c["B"]), n).astype(np.int32)
        path = np.full((c["B"], c["keep"]), -1, np.int32)
        for b in range(c["B"]):
            path[b, 0] = 0
            path[b, 1:kept[b]] = 1 + np.sort(rng.permutation(n[b] - 1)[:kept[b] - 1])
        return p, n, path, kept
    if c["kind"] != "attn":
        return np.zeros(c["B"], np.int32), n
    return _spread(rng, c["p_min"], c["p"], c["B"]), n


def _ceil16(x):
    return -(-x // BS)


def work(c):
    kind = c["kind"]
    if kind == "compact":
        _, _, path, kept = _lens(c)
        moved = int((path > np.arange(path.shape[1])[None, :]).sum())
        return {"bytes": moved * c["L"] * c["Hkv"] * c["D"] * 8 + 4 * int(kept.sum()) + 8 * c["B"], "flops": 0}
    p, n = (x.astype(np.int64) for x in _lens(c))
    T = int(n.sum())
    if kind == "tree":
        return {"bytes": T * (8 + 8 * c["words"]) + 8 * c["B"], "flops": 0}
    if kind == "verify":
        # The last node's row, and the draft's (nearly every walk ends behind a rejected token).
        return {"bytes": c["B"] * c["V"] * (8 if c["drawn"] and c["n"] > 1 else 4) + 12 * T, "flops": 0}
    seen = n * p + n * (n + 1) // 2                  # (a chain's; the masks decide how much of the tree a row sees)
    return {"bytes": int((p + n).sum()) * c["Hkv"] * c["D"] * 4 + T * (c["Hq"] * c["D"] * 4 + 8 * c["words"]),
            "flops": int(seen.sum()) * 4 * c["D"] * c["Hq"]}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _tables(blocks, nb, seed):
    """A table with blocks[b] distinct random pool blocks per row (the rest -1) of a pool of nb
    blocks."""
    perm = np.random.Generator(np.random.PCG64(seed)).permutation(nb).astype(np.int32)
    bt = np.full((len(blocks), max(1, int(blocks.max()))), -1, np.int32)
    at = np.arange(bt.shape[1])[None, :] < blocks[:, None]
    bt[at] = perm[:int(blocks.sum())]
    return bt


def _parents(c, n, seed):
    """A tree per sequence: every node follows one of the `back` nodes before it."""
    rng = np.random.Generator(np.random.PCG64(seed))
    out = []
    for s in n:
        i = np.arange(int(s))
        par = i - 1 - rng.integers(0, c["back"], size=int(s))
        out.append(np.where(i == 0, -1, np.maximum(par, 0)))
    return np.concatenate(out + [np.zeros(0)]).astype(np.int32)


def _visible(cu, parents, words):
    """Bit k of row i: node k is i or one of its ancestors."""
    vis = np.zeros((len(parents), words), np.uint64)
    for b in range(len(cu) - 1):
        for i in range(int(cu[b + 1] - cu[b])):
            t, par = cu[b] + i, parents[cu[b] + i]
            if par >= 0:
                vis[t] = vis[cu[b] + par]
            vis[t, i // 64] |= np.uint64(1 << (i % 64))
    return vis.view(np.int64)


def prepare(c, seed):
    kind = c["kind"]
    gen = _gen(seed)
    st = dict(c, own=own)
    if kind == "compact":
        p, n, path, kept = _lens(c)
        blocks = _ceil16(p + n)
        nb = int(blocks.sum()) + 8
        # [layer][K, V]; the layers' pools are parts of it
        kv = torch.empty(c["L"], 2, nb, c["Hkv"], BS * c["D"], dtype=torch.bfloat16, device=DEV)
        for layer in kv:
            layer.copy_(_normal(gen, *layer.shape))
        st.update(kv=kv, bt=_dev(_tables(blocks, nb, seed)), p=_dev(p), path=_dev(path), kept=_dev(kept))
    else:
        p, n = _lens(c)
        cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        T = int(cu[-1])
        parents = _parents(c, n, seed)
        if kind != "attn":                        # no work goes by the cached tokens: any count does
            p = np.random.Generator(np.random.PCG64(seed)).integers(0, 8000, size=c["B"]).astype(np.int32)
        st.update(h_p=p, h_cu=cu, h_parents=parents, T=T, p=_dev(p), cu=_dev(cu), parents=_dev(parents))
    if kind == "tree":
        st.update(visible=torch.empty(T, c["words"], dtype=torch.int64, device=DEV),
                  positions=torch.empty(T, dtype=torch.int32, device=DEV))
    elif kind == "attn":
        D, Hq, Hkv = c["D"], c["Hq"], c["Hkv"]
        blocks = _ceil16(p + n)
        nb = int(blocks.sum()) + 8
        st.update(bt=_dev(_tables(blocks, nb, seed)), pool_k=_normal(gen, nb, Hkv, BS * D),
                  pool_v=_normal(gen, nb, Hkv, BS * D), q=_normal(gen, T, Hq, D),
                  visible=_dev(_visible(cu, parents, c["words"])))
        st["out"] = torch.empty_like(st["q"])
    elif kind == "verify":
        st.update(_probabilities(c, gen, cu, parents))
        st.update(path=torch.empty(c["B"], c["n"], dtype=torch.int32, device=DEV),
                  kept=torch.empty(c["B"], dtype=torch.int32, device=DEV),
                  token=torch.empty(c["B"], dtype=torch.int32, device=DEV),
                  ctx=torch.empty(c["B"], dtype=torch.int32, device=DEV))
    if own:
        _prepare_own(st)
    return st


def _probabilities(c, gen, cu, parents):
    """The target's and the draft's distributions behind every node, which differ as a small
    model's do from a large one's, and the drafted tokens: drawn from the draft's distribution
    behind their parent, or (drawn = 0) its most likely ones, each sibling another."""
    T, V = len(parents), c["V"]
    target = torch.empty(T, V, device=DEV)
    draft = torch.empty(T, V, device=DEV)
    tokens = torch.zeros(T, dtype=torch.int32, device=DEV)
    # the rank of every node among its siblings
    rank, seen = np.zeros(T, np.int64), {}
    first = np.repeat(cu[:-1], np.diff(cu))
    at = np.maximum(parents, 0) + first
    for t in range(T):
        rank[t] = seen.get(at[t], 0) if parents[t] >= 0 else 0
        seen[at[t]] = rank[t] + (1 if parents[t] >= 0 else 0)
    rank, at = _dev(rank), _dev(at.astype(np.int64))
    for a in range(0, T, 256):
        e = min(T, a + 256)
        logits = 3.5 * torch.randn(e - a, V, generator=gen, device=DEV)
        target[a:e] = torch.softmax(logits, -1)
        draft[a:e] = torch.softmax(0.97 * logits + 0.8 * torch.randn(e - a, V, generator=gen, device=DEV), -1)
    for a in range(0, T, 256):
        e = min(T, a + 256)
        if c["drawn"]:
            pick = torch.multinomial(draft[at[a:e]], 1, generator=gen)
        else:
            k = min(V, int(rank.max()) + 1)
            pick = torch.topk(draft[at[a:e]], k, dim=-1).indices.gather(1, rank[a:e, None])
        tokens[a:e] = pick[:, 0].to(torch.int32)
    uniforms = torch.rand(T, generator=gen, device=DEV)
    return dict(target=target, draft=draft if c["drawn"] else None, tokens=tokens, uniforms=uniforms)


def _prepare_own(st):
    """What a serving program keeps beside its tensors: the pools' handles and the workspaces."""
    from paper_2603_23049_amd import pcr
    kind = st["kind"]
    if kind == "attn":
        st["pool"] = pcr.KVPool(st["pool_k"], st["pool_v"], st["Hkv"], st["D"])
        nbytes = pcr.tree_attn_workspace_bytes(st["B"], st["T"], st["Hq"], st["Hkv"], st["D"],
                                               int((st["h_p"] + np.diff(st["h_cu"])).max()))
        st["ws"] = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=DEV)
    elif kind == "verify":
        nbytes = pcr.verify_drafts_workspace_bytes(st["B"], st["T"], st["V"])
        st["ws"] = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=DEV)
    elif kind == "compact":
        st["pools"] = pcr.KVLayers([pcr.KVPool(layer[0], layer[1], st["Hkv"], st["D"]) for layer in st["kv"]])


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(st):
    return (_run_own if own else _run_plain)(st)


def _run_own(st):
    from paper_2603_23049_amd import pcr
    kind = st["kind"]
    if kind == "tree":
        pcr.draft_tree(st["cu"], st["parents"], st["p"], st["visible"], st["positions"])
        return [st["visible"], st["positions"]]
    if kind == "attn":
        pcr.tree_attn(st["q"], st["pool"], st["bt"], st["p"], st["cu"], st["h_p"], st["h_cu"], st["visible"], st["Hq"],
                      st["out"], workspace=st["ws"])
        return [st["out"]]
    if kind == "verify":
        pcr.verify_drafts(st["cu"], st["parents"], st["tokens"], st["target"], st["draft"], st["uniforms"], st["p"],
                          st["path"], st["kept"], st["token"], st["ctx"], workspace=st["ws"])
        return [st["path"], st["kept"], st["token"], st["ctx"]]
    pcr.compact_kv(st["pools"], st["bt"], st["p"], st["path"], st["kept"])
    return [st["kv"]]


def _run_plain(st):
    return {"tree": _plain_tree, "attn": _plain_attn, "verify": _plain_verify, "compact": _plain_compact}[st["kind"]](st)


def _rows(cu, n):
    """[B][n]: every sequence's rows, and which of them it has."""
    i = torch.arange(n, device=cu.device)[None, :]
    rows = cu[:-1, None].long() + i
    return rows, rows < cu[1:, None]


def _plain_tree(st):
    B, n, W = st["B"], st["n"], st["words"]
    rows, live = _rows(st["cu"], n)
    rows = rows.clamp(max=st["T"] - 1)
    par = torch.where(live, st["parents"][rows].long(), torch.full_like(rows, -1))
    # node i reaches k in any number of steps: (I + A)^n, squared
    i = torch.arange(n, device=DEV)
    reach = ((par[:, :, None] == i) | (i[:, None] == i)).float()
    for _ in range(max(1, (n - 1).bit_length())):
        reach = (torch.bmm(reach, reach) > 0).float()
    reach = reach.bool()
    bits = torch.zeros(B, n, W * 64, dtype=torch.int64, device=DEV)
    bits[:, :, :n] = reach
    words = (bits.view(B, n, W, 64) << torch.arange(64, device=DEV)).sum(-1)
    pos = st["p"].long()[:, None] + reach.sum(-1) - 1
    st["visible"].copy_(words[live])
    st["positions"].copy_(pos[live])
    return [st["visible"], st["positions"]]


def _plain_attn(st):
    B, n, D, Hq, Hkv = st["B"], st["n"], st["D"], st["Hq"], st["Hkv"]
    G, keys = Hq // Hkv, st["bt"].shape[1] * BS
    rows, live = _rows(st["cu"], n)
    rows = rows.clamp(max=st["T"] - 1)
    bt = st["bt"].long().clamp(min=0)
    k = st["pool_k"][bt].float().view(B, -1, Hkv, BS, D).permute(0, 2, 4, 1, 3).reshape(B * Hkv, D, keys)
    v = st["pool_v"][bt].float().view(B, -1, Hkv, D, BS).permute(0, 2, 1, 4, 3).reshape(B * Hkv, keys, D)
    q = st["q"][rows].float().view(B, n, Hkv, G, D).transpose(1, 2).reshape(B * Hkv, n * G, D)
    # what every row sees
    j = torch.arange(keys, device=DEV)[None, :] - st["p"].long()[:, None]          # [B][keys]: node, below 0 cached
    node = j.clamp(0, st["words"] * 64 - 1)[:, None, :].expand(B, n, keys)
    word = st["visible"][rows].gather(2, node // 64)
    sees = (((word >> (node % 64)) & 1) != 0) & (j < (st["cu"][1:] - st["cu"][:-1])[:, None])[:, None, :]
    sees = (sees | (j < 0)[:, None, :])[:, None, :, None, :].expand(B, Hkv, n, G, keys).reshape(B * Hkv, n * G, keys)
    s = (torch.bmm(q, k) * D ** -0.5).masked_fill_(~sees, -math.inf)
    w = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-3e38))
    o = torch.bmm(w, v) / w.sum(-1, keepdim=True).clamp(min=1e-30)
    o = o.view(B, Hkv, n, G, D).transpose(1, 2).reshape(B, n, Hq, D)
    st["out"].copy_(o[live])
    return [st["out"]]


def _plain_verify(st):
    B, n, V, T = st["B"], st["n"], st["V"], st["T"]
    target, draft = st["target"], st["draft"]
    rows, live = _rows(st["cu"], n)
    rows = rows.clamp(max=T - 1)
    par, tok, u = st["parents"][rows], st["tokens"][rows].long(), st["uniforms"][rows].double()
    first, seq = rows[:, 0], torch.arange(B, device=DEV)
    at = torch.zeros(B, dtype=torch.int64, device=DEV)            # the node that the walk stands on
    a = torch.zeros(B, dtype=torch.float64, device=DEV)
    z = torch.ones(B, dtype=torch.float64, device=DEV)
    gone = torch.zeros(B, V, dtype=torch.bool, device=DEV)        # refused tokens of a draft without probabilities
    path = torch.zeros(B, n, dtype=torch.bool, device=DEV)
    path[:, 0] = live[:, 0]

    def rest():
        """What is left of the last node's distribution."""
        p = target[first + at].double()
        if draft is None:
            return p.masked_fill_(gone, 0.0)
        return (p - a[:, None] * draft[first + at].double()).clamp_(min=0.0)

    for i in range(1, n):
        x, here = tok[:, i], live[:, i] & (par[:, i] == at)
        p = target[first + at, x].double()
        if draft is None:
            w, ask = torch.where(gone[seq, x], 0.0, p), u[:, i] * z
        else:
            q = draft[first + at, x].double()
            w, ask = (p - a * q).clamp(min=0.0), u[:, i] * q * z
        yes, no = here & (ask < w), here & ~(ask < w)
        path[:, i] = yes
        at = torch.where(yes, i, at)
        if draft is None:
            gone[seq, x] |= no
            gone &= ~yes[:, None]
            z = torch.where(yes, 1.0, torch.where(no, z - w, z))
        else:
            a = torch.where(yes, 0.0, torch.where(no, a + z, a))
            z = torch.where(yes, 1.0, torch.where(no, rest().sum(-1), z))
    r = rest()
    r = torch.where((r.sum(-1) > 0)[:, None], r, target[first + at].double())
    most = u[:, 0] * r.sum(-1)
    last = V - 1 - (r > 0).flip(-1).to(torch.int8).argmax(-1)
    token = torch.minimum((r.cumsum(-1) <= most[:, None]).sum(-1), last)
    kept = path.sum(-1)
    order = torch.where(path, torch.arange(n, device=DEV), n).sort(-1).values
    st["path"].copy_(torch.where(order < n, order, -1))
    st["kept"].copy_(kept)
    st["token"].copy_(torch.where(live[:, 0], token, -1))
    st["ctx"].copy_(st["p"] + kept)
    return [st["path"], st["kept"], st["token"], st["ctx"]]


def _plain_compact(st):
    D, Hkv, L = st["D"], st["Hkv"], st["L"]
    i = torch.arange(st["path"].shape[1], device=DEV)[None, :]
    moves = (i < st["kept"][:, None]) & (st["path"] > i)
    b, k = moves.nonzero(as_tuple=True)
    src, dst = st["p"].long()[b] + st["path"].long()[b, k], st["p"].long()[b] + k
    sb, db = st["bt"].long()[b, src // BS], st["bt"].long()[b, dst // BS]
    kk, vv = st["kv"][:, 0].view(L, -1, Hkv, BS, D), st["kv"][:, 1].view(L, -1, Hkv, D, BS)
    k_rows, v_rows = kk[:, sb, :, src % BS], vv[:, sb, :, :, src % BS]
    kk[:, db, :, dst % BS] = k_rows
    vv[:, db, :, :, dst % BS] = v_rows
    return [st["kv"]]


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------

def exact(c, seed):
    kind = c["kind"]
    if kind in ("tree", "verify"):
        return None                       # whole numbers
    st = prepare(c, seed)
    return [_exact_attn(c, st) if kind == "attn" else _exact_compact(c, st)]


def _exact_attn(c, st):
    """One (sequence, query head) at a time; what a node sees by following its parents."""
    D, Hq, G = c["D"], c["Hq"], c["Hq"] // c["Hkv"]
    res = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    for b in range(c["B"]):
        p, t0, t1 = int(st["h_p"][b]), int(st["h_cu"][b]), int(st["h_cu"][b + 1])
        n = t1 - t0
        if n == 0:
            continue
        hide = np.ones((n, p + n), bool)
        hide[:, :p] = False
        for i in range(n):
            k = i
            while k >= 0:
                hide[i, p + k] = False
                k = int(st["h_parents"][t0 + k])
        hide = _dev(hide)
        blocks = st["bt"][b, :_ceil16(p + n)].long()
        for g in range(c["Hkv"]):
            k = st["pool_k"][blocks, g].reshape(-1, D)[:p + n].double()
            v = st["pool_v"][blocks, g].reshape(-1, D, BS).transpose(1, 2).reshape(-1, D)[:p + n].double()
            for h in range(g * G, (g + 1) * G):
                s = (st["q"][t0:t1, h].double() @ k.t()) / math.sqrt(D)
                res[t0:t1, h] = torch.softmax(s.masked_fill(hide, -math.inf), dim=1) @ v
    return res


def _exact_compact(c, st):
    """Token after token, in the order of the path."""
    kv = st["kv"].double()
    D, Hkv, L = c["D"], c["Hkv"], c["L"]
    k, v = kv[:, 0].view(L, -1, Hkv, BS, D), kv[:, 1].view(L, -1, Hkv, D, BS)
    p, path, kept, bt = (st[x].tolist() for x in ("p", "path", "kept", "bt"))
    for b in range(c["B"]):
        for i in range(kept[b]):
            s, d = p[b] + path[b][i], p[b] + i
            if s != d:
                k[:, bt[b][d // BS], :, d % BS] = k[:, bt[b][s // BS], :, s % BS].clone()
                v[:, bt[b][d // BS], :, :, d % BS] = v[:, bt[b][s // BS], :, :, s % BS].clone()
    return kv
