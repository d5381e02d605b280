"""CPU: register use of the kernels around the pool (block tables, rotary positions, cross
attention), from the compiler's resource report for gfx950: no kernel spills or uses scratch,
and what the decode-shaped ones hold fits the waves their plan counts as resident."""
import os

import pytest

from test_kernel_resources import HIPCC, _resources

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")


@pytest.mark.parametrize("src", ["blocks.hip", "rope.hip", "cross.hip", "cross_rows.hip"])
def test_no_spills(src):
    res = _resources(src)
    assert res
    for name, r in res.items():
        assert r["VGPRs Spill"] == 0 and r["SGPRs Spill"] == 0 and r["ScratchSize"] == 0, (name, r)


def test_cross_rows_waves_are_resident():
    for name, r in _resources("cross_rows.hip").items():
        if "cross_rows_kernel" in name:
            assert r["Occupancy"] >= (2 if "ILi64" in name else 1), (name, r)
