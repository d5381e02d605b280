"""CPU: when verification keeps the target's distribution. The rule of pcr_verify_drafts in exact fractions over all
drafts of a node's two or three children: exact where they are drawn independently, and where no draft
probabilities are given; not where they are drawn without replacement."""
from fractions import Fraction as F
from itertools import permutations, product

import pytest

P = [F(1, 2), F(1, 5), F(1, 5), F(1, 10)]
Q = [F(1, 10), F(3, 10), F(2, 5), F(1, 5)]


def _new_token(p, q, children):
    """Distribution of the first new token: the kept child's, or the one drawn after all were refused."""
    out, left = [F(0)] * len(p), F(1)              # left: chance that every child so far was refused
    a, Z, r = F(0), F(1), list(p)
    for x in children:
        w = r[x]
        ask = (q[x] if q else F(1)) * Z            # kept where u * ask < w
        keep = F(0) if w <= 0 else min(F(1), w / ask)
        out[x] += left * keep
        left *= 1 - keep
        if left == 0:
            return out
        if q:
            a += Z
            r = [max(y - a * z, F(0)) for y, z in zip(p, q)]
            Z = sum(r)
        else:
            Z -= w
            r[x] = F(0)
    S = sum(r)
    return [o + left * y / S for o, y in zip(out, r)]


def _over(drafts, q, p=P):
    total = [F(0)] * len(p)
    for chance, children in drafts:
        total = [t + chance * y for t, y in zip(total, _new_token(p, q, children))]
    return total


@pytest.mark.parametrize("n", [1, 2, 3])
def test_children_drawn_independently(n):
    drafts = []
    for c in product(range(4), repeat=n):
        chance = F(1)
        for x in c:
            chance *= Q[x]
        drafts.append((chance, c))
    assert sum(c for c, _ in drafts) == 1
    assert _over(drafts, Q) == P


@pytest.mark.parametrize("children", [(2,), (2, 1), (2, 1, 3), (0, 0, 1), (3, 3)])
def test_without_probabilities(children):
    assert _over([(F(1), children)], None) == P


def test_children_drawn_without_replacement_are_not_the_targets():
    """Two children: the second, drawn from q without the first, is judged as if drawn from all of q. What the first one's
    refusal leaves, max(p - q, 0), is one token of P, which then comes whatever the second is; of P2 it is two."""
    P2, Q2 = [F(2, 5), F(2, 5), F(1, 10), F(1, 10)], [F(1, 10), F(1, 5), F(2, 5), F(3, 10)]
    for p, q, same in ((P, Q, True), (P2, Q2, False)):
        drafts = [(q[x] * q[y] / (1 - q[x]), (x, y)) for x, y in permutations(range(4), 2)]
        assert sum(c for c, _ in drafts) == 1
        assert (_over(drafts, q, p) == p) == same
        assert _over(drafts, None, p) == p
        assert _over([(q[x] * q[y], (x, y)) for x, y in product(range(4), repeat=2)], q, p) == p
