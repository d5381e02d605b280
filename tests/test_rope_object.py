"""CPU: a rotation's arrays live as long as the rotation, whatever becomes of its attributes: the
library reads them at every call."""
import gc
import weakref

import numpy as np

from paper_2603_23049_amd import pcr


def test_arrays_outlive_the_attributes():
    f = np.arange(8, dtype=np.float32)
    rope = pcr.Rope(f, np.zeros(8, np.int32))
    arrays = [weakref.ref(rope.inv_freq), weakref.ref(rope.pair_axis)]
    where = [rope._c.inv_freq, rope._c.pair_axis]
    rope.inv_freq = np.ones(8, np.float32)
    rope.pair_axis = None
    gc.collect()
    assert [a() is not None for a in arrays] == [True, True]
    assert [a().ctypes.data for a in arrays] == where and np.array_equal(arrays[0](), f)
    f[:] = 9                                   # (copied when the rotation was made)
    assert arrays[0]()[1] == 1
