"""GPU: which rows of the probabilities verification depends on: those of the nodes that its walk comes to."""
import numpy as np
import pytest

from test_gpu_verify import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,V,back", [([9, 25, 1, 70], 300, 5), ([13, 20], 20011, 4), ([12, 30, 11], 50000, 6)])
def test_rows_away_from_the_walk_change_nothing(n, V, back):
    c = Case(n, V, True, 40 + V, back)
    path, kept, _, _ = want = c.want()
    came = np.zeros(c.T, bool)
    for b in range(c.B):
        came[c.cu[b] + path[b, :kept[b]]] = True
    has_child = np.zeros(c.T, bool)
    for b in range(c.B):
        for i in range(1, int(c.n[b])):
            has_child[c.cu[b] + c.parents[c.cu[b] + i]] = True
    assert (~came).any() and (came & ~has_child).sum() + (~came & has_child).sum() > 0
    c.target[~came] = np.nan
    c.draft[~(came & has_child)] = np.nan
    for got, w in zip(c.run(stride=1), want):
        assert np.array_equal(got, w)
