"""CPU: the order of a ragged prefill launch on 1, 2 and 4 kv heads (a device of 256 compute units): the XCDs that
share a head take parts of its items where that balances them, and the given order where one long
sequence leaves the parts unequal and the order is estimated to be no slower."""
import ctypes
import random

import numpy as np
import pytest

from paper_2603_23049_amd import pcr

N_CU = 256


def _parts(p, s, Hq, Hkv, d, rpw=128):
    """Parts of a head's items: 8 / Hkv, or 1 for the given order."""
    f = pcr.lib()._ZN3pcr18prefill_attn_partsEPKiiS1_S1_iiiii          # internal: pcr::prefill_attn_parts
    f.restype, f.argtypes = ctypes.c_int32, [ctypes.c_void_p, ctypes.c_int32] + [ctypes.c_void_p] * 2 + [ctypes.c_int32] * 5
    p, cu = np.asarray(p, np.int32), np.concatenate([[0], np.cumsum(s)]).astype(np.int32)
    seq = np.argsort(-(p + np.asarray(s)), kind="stable").astype(np.int32)
    return f(seq.ctypes.data, len(p), p.ctypes.data, cu.ctypes.data, Hq, Hkv, d, rpw, N_CU)


# (measured with the given order / in parts, us)
@pytest.mark.parametrize("p,s,Hq,Hkv,d", [
    ([8000] * 6 + [2000, 0], [16] * 6 + [900, 2000], 16, 2, 128),      # 85 / 108
    ([8000] * 20 + [0], [16] * 20 + [1600], 32, 4, 64),                 # 77 / 85
    ([8000] * 10 + [0], [16] * 10 + [3000], 32, 4, 64),                 # 94 / 104
    ([8000] * 20 + [0], [16] * 20 + [1600], 32, 4, 128),                # 103 / 111
    ([8000] * 20 + [0], [18] * 20 + [1600], 28, 4, 128),                # 103 / 110
])
def test_one_long_prompt_behind_short_ones_keeps_the_order(p, s, Hq, Hkv, d):
    assert _parts(p, s, Hq, Hkv, d) == 1


@pytest.mark.parametrize("p,s,Hq,Hkv,d", [
    ([4000] * 30 + [0], [16] * 30 + [1000], 32, 4, 128),                # 69 / 57
    ([6000] * 40 + [0], [16] * 40 + [4000], 16, 2, 128),                # 165 / 132
    ([8000] * 20 + [0, 100], [16] * 20 + [700, 650], 32, 4, 128),       # 108 / 99: equal parts
])
def test_parts_that_gain_stay(p, s, Hq, Hkv, d):
    assert _parts(p, s, Hq, Hkv, d) == 8 // Hkv


def test_equal_parts_are_taken():
    rnd = random.Random(4)
    for _ in range(200):
        Hkv, d = rnd.choice([1, 2, 4]), rnd.choice([64, 128])
        n = 8 // Hkv * rnd.randint(2, 9)
        p = [rnd.randint(0, 8000) for _ in range(n)]
        p[:2] = [0, 8000]
        assert _parts(p, [60] * n, 8 * Hkv, Hkv, d) == 8 // Hkv         # a count of items that divides
        assert _parts([500] * n, [60] * n, 8 * Hkv, Hkv, d) == 1        # one length: any order
