"""CPU: how tree attention of few rows is cut on a device of 256 compute units: that the cases of the GPU
tests take every form the library has, that no plan needs more workspace than the size query says,
and what the kernels hold."""
import ctypes
import os
import random
import re

import pytest

import test_gpu_tree_forms as forms
from paper_2603_23049_amd import pcr
from test_kernel_resources import HIPCC, _resources

N_CU = 256
WHOLE, PARTS, EVEN = range(3)


class Plan(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in ("runs", "waves", "parts", "slots")]


class Cost(ctypes.Structure):
    _fields_ = [(f, ctypes.c_float) for f in ("cu", "parts", "even")] + [("waves", ctypes.c_int32)]


def _plan(steps, pairs, longest, d, rows):
    f = pcr.lib()._ZN3pcr9rows_planEllliiRKNS_8RowsCostE          # internal: pcr::rows_plan
    f.restype, f.argtypes = Plan, [ctypes.c_int64] * 3 + [ctypes.c_int32] * 2 + [ctypes.POINTER(Cost)]
    cost = Cost(0.29 if d == 128 else 0.15, 11.0, 1.25 if rows > 16 else 1.0, 4)  # tree.hip's
    return f(steps, pairs, longest, d, N_CU, ctypes.byref(cost))


def _form(p, n, Hq, Hkv, d):
    rows = n * Hq // Hkv
    assert rows <= 32
    steps = [-(-(x + n) // 32) for x in p]
    plan = _plan(sum(steps) * Hkv, len(p) * Hkv, max(steps), d, rows)
    return d, plan.waves, WHOLE if plan.parts == 1 else PARTS if plan.parts else EVEN, 1 if rows <= 16 else 2


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_every_form_is_tested_and_resident():
    built = {}
    for name, r in _resources("tree_rows.hip").items():
        assert r["VGPRs Spill"] == 0 and r["ScratchSize"] == 0, (name, r)
        m = re.search(r"cross_rows_kernelILi(\d+)ELi(\d+)ELi(\d)ELi(\d)E", name)
        if m:
            built[tuple(map(int, m.groups()))] = r
    assert len(built) == 24
    assert {_form(*f) for f in forms.FORMS} == set(built)
    for (d, waves, cut, tiles), r in built.items():
        assert r["Occupancy"] >= (1 if d == 128 else 2), (d, waves, cut, tiles, r)   # as the plan counts them


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
@pytest.mark.parametrize("src", ["draft.hip", "verify.hip", "tree.hip"])
def test_no_spills(src):
    for name, r in _resources(src).items():
        assert r["VGPRs Spill"] == 0 and r["ScratchSize"] == 0, (name, r)


def test_workspace_size_covers_every_plan():
    rnd = random.Random(6)
    max_slots = pcr.lib()._ZN3pcr20cross_rows_max_slotsEii
    max_slots.restype, max_slots.argtypes = ctypes.c_int64, [ctypes.c_int32] * 2
    seen = set()
    for _ in range(20000):
        d, Hkv, B, rows = rnd.choice([64, 128]), rnd.randint(1, 16), rnd.randint(1, rnd.choice([8, 300, 5000])), rnd.randint(1, 32)
        live, longest = rnd.randint(1, B), rnd.randint(1, rnd.choice([4, 40, 2000, 50000]))
        steps = rnd.randint(longest + live - 1, longest * live) * Hkv
        p = _plan(steps, B * Hkv, longest, d, rows)
        seen.add(min(p.parts, 2))
        if p.parts == 1 or p.runs == 1:
            continue                      # no pair is cut
        assert p.slots <= min(B * Hkv * longest, max_slots(d, N_CU))
    assert seen == {0, 1, 2}
