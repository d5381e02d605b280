"""GPU: verification by rounds: walks that end in every round and after the last one, workgroups whose waves sum
several tiles, tiles of several pieces. (test_verify_plan.py holds the cases to the forms they are here for.)"""
import numpy as np
import pytest

import treeref
from test_gpu_verify import Case

pytestmark = pytest.mark.gpu

# name: nodes of each sequence, vocabulary, with the draft's probabilities, back, away (how far the draft is from the target)
CASES = {
    "four rounds": ([14, 40, 0, 11, 25, 1, 64, 18, 12, 30], 50021, True, 6, 2.5),
    "four rounds, chains": ([12] * 9, 49500, True, 1, 1.0),
    "four rounds, bushes": ([20, 17, 33], 66000, True, 200, 3.0),
    "four rounds, many sequences": ([10, 16, 1, 13, 12] * 20, 50000, True, 5, 2.0),
    "two rounds": ([9, 7, 6, 9], 49300, True, 3, 2.0),
    "two rounds, more sequences": ([9, 8, 6, 7, 9, 9, 6, 8] * 2, 49153, True, 3, 2.0),
    "one round, many sequences": ([5, 3] * 60, 41000, True, 2, 1.5),
    "one round, no probabilities, many sequences": ([9, 0, 4] * 40, 41000, False, 3, 1.0),
    "two pieces, one round": ([3, 4], 4194305, True, 2, 1.0),
    "two pieces, four rounds": ([12], 4200007, True, 12, 3.0),
    "two pieces, no probabilities": ([4], 4198401, False, 3, 1.0),
}


def case(name):
    n, V, drawn, back, away = CASES[name]
    return Case(n, V, drawn, 900 + sum(n), back, sharp=1.0, away=away)


def passes(c):
    """Sums that each sequence's walk takes: one for every refusal with probabilities, and one of the last row
    where none of them was of that row as it was left."""
    path, kept, _, _ = c.want()
    out = []
    for b in range(c.B):
        if c.n[b] == 0:
            continue
        t0, way, n, u = int(c.cu[b]), path[b, :kept[b]].tolist(), 0, 0
        for step, u in enumerate(way):
            kids = [i for i in range(u + 1, int(c.n[b])) if c.parents[t0 + i] == u]
            stays = way[step + 1] if step + 1 < len(way) else None
            refused = kids.index(stays) if stays is not None else len(kids) if len(way) < c.cap else 0
            n += refused if c.draft is not None else 0
            if stays is None and (c.draft is None or refused == 0):
                n += 1
        out.append(n)
    return out


@pytest.mark.parametrize("name", list(CASES))
def test_rounds(name):
    c = case(name)
    want = c.want()
    for _ in range(2):
        for got, w, what in zip(c.run(), want, ("path", "accepted_lens", "next_tokens", "context_lens")):
            assert np.array_equal(got, w), (what, got, w)


def test_a_sequence_alone_or_among_others():
    """The rounds differ with the batch (four, two, one, none for short vocabularies): the tokens do not."""
    c = case("four rounds")
    among = c.run()
    for b in range(c.B):
        if c.n[b] == 0:
            continue
        t = slice(int(c.cu[b]), int(c.cu[b + 1]))
        one = object.__new__(Case)
        one.n, one.V, one.B, one.cap = c.n[b:b + 1], c.V, 1, c.cap
        one.cu, one.T = np.array([0, int(c.n[b])]), int(c.n[b])
        one.parents, one.tokens, one.uniforms = c.parents[t], c.tokens[t], c.uniforms[t]
        one.target, one.draft, one.p = c.target[t], c.draft[t], c.p[b:b + 1]
        for got, w in zip(one.run(), among):
            assert np.array_equal(got[0], w[b])


def test_reference_counts_passes():
    """(of the counting above: a walk that refuses nothing takes one sum)"""
    c = Case([7] * 8, 500, True, 3, back=1)
    c.draft = c.target
    assert passes(c) == [1] * 8 and (treeref.verify(c.cu, c.parents, c.tokens, c.target, c.draft, c.uniforms, c.p,
                                                    c.cap)[1] == 7).all()
