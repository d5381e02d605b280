"""GPU: cross attention of few rows in the forms that test_gpu_cross_cuts does not take (which
those are, test_cross_plan says on the CPU): even runs of four waves and whole pairs of two at 64
dims, and pairs of more parts than a merge takes at a time; and keys whose products overflow, wherever the work is cut. The
tolerance is test_gpu_cross's."""
import numpy as np
import pytest
import torch

from test_gpu_cross import _case, _close, _run

pytestmark = pytest.mark.gpu
BS = 16

FORMS = [
    ([16000, 2000, 1000], [1, 1, 1], 8, 8, 64),              # even runs of four waves
    ([40000], [1], 1, 1, 64), ([40000], [3], 4, 1, 64),      # 156 runs in one pair
    ([20000], [2], 2, 1, 128),                               # 78
    ([25600], [1], 2, 1, 64),                                # 100 equal parts of one pair
    (list(range(30, 330)), [1] * 300, 4, 2, 64),             # whole pairs of two waves
]


@pytest.mark.parametrize("keys,rows,Hq,Hkv,d", FORMS)
def test_forms(keys, rows, Hq, Hkv, d):
    c = _case(keys, rows, Hq, Hkv, d, sum(keys) + d)
    got = _run(*c, Hkv, d)
    _close(got, *c, Hkv, d)
    assert torch.equal(got, _run(*c, Hkv, d))


@pytest.mark.parametrize("keys,rows,Hq,Hkv,d", [
    ([40], [2], 8, 2, 64), ([2438, 2438], [1, 2], 14, 2, 128), ([3000, 70, 900, 1601] * 15, [1] * 60, 4, 1, 128),
    ([13000, 2000, 1000], [1, 1, 1], 8, 8, 128), ([300, 65], [40, 3], 8, 2, 64), ([6000, 7000], [20, 1], 8, 1, 128)])
@pytest.mark.parametrize("low", ["first", "last", "even steps"])
def test_keys_whose_products_overflow_weigh_nothing(keys, rows, Hq, Hkv, d, low):
    """Keys of -3e38 under queries of one sign: their scores are -inf in 32 bits and far below every
    other in 64, so they weigh nothing in either."""
    q, pk, pv, bt, n, cu = _case(keys, rows, Hq, Hkv, d, 5, poison=False)
    q = q.abs()
    k = pk.view(-1, Hkv, BS, d)
    for b, nb in enumerate(keys):
        t = np.arange(nb)
        t = t[{"first": t < nb // 2, "last": t >= (nb + 1) // 2, "even steps": t // 32 % 2 == 0}[low]]
        if len(t) < nb:
            k[torch.from_numpy(bt[b][t // BS].astype(np.int64)), :, torch.from_numpy(t % BS)] = -3e38
    _close(_run(q, pk, pv, bt, n, cu, Hkv, d), q, pk, pv, bt, n, cu, Hkv, d)
