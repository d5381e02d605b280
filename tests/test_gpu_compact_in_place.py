"""GPU: path entries that are in their place end no moves, whatever the table holds for their slots."""
import numpy as np
import pytest

from test_gpu_compact import _case, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hkv,d", [(3, 64), (2, 128)])
@pytest.mark.parametrize("bad", [-1, 10 ** 6, 2 ** 31 - 1])
def test_in_place_entries_in_bad_blocks(bad, Hkv, d):
    p = [0, 32, 5]
    _, bt, kv = _case(p, [60] * 3, Hkv, d, 2, 11)
    path = np.tile(np.array(list(range(16)) + [20, 25, 40]), (3, 1))
    bt[0, 0] = bt[1, 2] = bad                    # the blocks of entries 0 to 15 of sequences 0 and 1
    bt[2, 1] = bad                               # sequence 2: the target of its entry 16 lies there, nothing moves
    _check(kv, bt, p, path, [19, 18, 19], Hkv, d)
