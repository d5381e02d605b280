"""CPU: what the rotations refuse because of its size alone: launches beyond 2^32 threads, and
rows that reach past every address, where an overlap could not be told."""
import ctypes

import numpy as np
import pytest

from paper_2603_23049_amd import pcr

UNS = pcr.PCR_ERR_UNSUPPORTED
A = 1 << 50          # addresses that are never read, far apart


def _rope(rd, axes=1):
    f = np.ones(rd // 2, np.float32)
    r = pcr._Rope(f.ctypes.data, None, rd, axes, 0, 1.0)
    r.keep = f
    return r


def _append(T, Hq, Hkv, d, k_stride=None, q_stride=None):
    pool, rope = pcr._Pool(A, A + (1 << 30), 4, 16, Hkv, d), _rope(d)
    return pcr.lib().pcr_rope_append_kv(ctypes.addressof(rope), ctypes.byref(pool), 2 * A, q_stride or Hq * d,
                                        4 * A, k_stride or Hkv * d, 6 * A, Hkv * d, 8 * A, T, 9 * A, T, Hq, 10 * A, None)


@pytest.mark.parametrize("T,Hq,Hkv,d", [(1 << 27, 32, 8, 64), (1 << 27, 16, 2, 128), (1 << 25, 64, 64, 128),
                                        ((1 << 22) + 5, 2048, 1, 64)])
def test_append_grid(T, Hq, Hkv, d):
    """Q takes one thread per 16 dims of 4 heads: T * Hq (64 dims) or 2 * T * Hq of them (128)."""
    assert _append(T, Hq, Hkv, d) == UNS and "threads" in pcr.last_error()


def test_rows_beyond_addresses():
    for kw in (dict(k_stride=1 << 40), dict(q_stride=1 << 40)):
        assert _append(1 << 24, 8, 2, 64, **kw) == UNS and "addresses" in pcr.last_error(), kw
    rope = _rope(64)
    for xs, os in ((1 << 40, 128), (128, 1 << 40), (1 << 40, 1 << 40)):
        # out's rows lie among x's: an end that wraps around would hide it
        assert pcr.lib().pcr_rope_rows(ctypes.addressof(rope), A, xs, 2 * A, 1 << 24, 1 << 24, 2, 64, 0, A + 4096, os,
                                       None) == UNS and "addresses" in pcr.last_error()
