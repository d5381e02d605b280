"""CPU: how cross attention of few rows is cut on a device of 256 compute units: that the cases of
the GPU tests take the forms they are there for, that between them they take every form the
library has, that no plan needs more workspace than the size query says, and that what the
plan counts as resident fits a compute unit."""
import ctypes
import os
import random
import re

import numpy as np
import pytest

import test_gpu_cross_cuts as cuts
import test_gpu_cross_forms as forms
from paper_2603_23049_amd import pcr
from test_kernel_resources import HIPCC, _resources

N_CU = 256
WHOLE, PARTS, EVEN = range(3)


class Plan(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in ("runs", "waves", "parts", "slots")]


def _plan(steps, pairs, longest, d):
    f = pcr.lib()._ZN3pcr15cross_rows_planElllii          # internal: pcr::cross_rows_plan
    f.restype, f.argtypes = Plan, [ctypes.c_int64] * 3 + [ctypes.c_int32] * 2
    return f(steps, pairs, longest, d, N_CU)


def _steps(n):
    return -(-n // 32)


def _form(keys, rows, Hq, Hkv, d):
    """((dims, waves, cut), most parts of a pair)."""
    live = [_steps(n) for n, r in zip(keys, rows) if r > 0]
    p = _plan(sum(live) * Hkv, len(keys) * Hkv, max(live), d)
    if p.parts == 1:
        return (d, p.waves, WHOLE), 1
    if p.parts > 1:
        return (d, p.waves, PARTS), max(-(-s // -(-s // p.parts)) for s in live if s)
    base, rem = divmod(sum(live) * Hkv, p.runs)
    begin = [u * base + min(u, rem) for u in range(p.runs + 1)]
    x, most = 0, 1
    for s in live:
        for _ in range(Hkv if s else 0):
            most = max(most, int(np.searchsorted(begin, x + s - 1, "right") - np.searchsorted(begin, x, "right")) + 1)
            x += s
    return (d, p.waves, EVEN), most


def _params(f):
    return next(m for m in f.pytestmark if m.name == "parametrize").args[1]


CUTS = [EVEN, EVEN, EVEN, EVEN, PARTS, PARTS, WHOLE, WHOLE, WHOLE, WHOLE, WHOLE, WHOLE, PARTS]


def test_cases_are_cut_as_they_say():
    got = [_form(*c) for c in _params(cuts.test_cuts)]
    assert [f[0][2] for f in got] == CUTS
    assert [f[0][1] for f in got[:4]] == [1, 1, 1, 4]
    got = [_form(*c) for c in forms.FORMS]
    assert got == [((64, 4, EVEN), 57), ((64, 4, EVEN), 156), ((64, 4, EVEN), 156), ((128, 4, EVEN), 78),
                   ((64, 4, PARTS), 100), ((64, 2, WHOLE), 1)]


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_every_form_is_tested_and_resident():
    built = {}
    for name, r in _resources("cross_rows.hip").items():
        m = re.search(r"cross_rows_kernelILi(\d+)ELi(\d+)ELi(\d)E", name)
        if m:
            built[tuple(map(int, m.groups()))] = r
    assert len(built) == 13
    tested = {_form(*c)[0] for c in _params(cuts.test_cuts) + forms.FORMS}
    assert tested == set(built)
    for (d, waves, cut), r in built.items():
        # waves of a compute unit in one round: a workgroup of each SIMD's registers (512 a lane), and of its LDS
        per_cu = 4 if d == 128 else 8
        regs = -(-(-(-r["VGPRs"] // 4) * 4 + r["AGPRs"]) // 8) * 8
        assert regs * (per_cu // 4) <= 512 and r["LDS Size"] * max(1, per_cu // waves) <= 160 * 1024, (d, waves, cut, r)
        assert r["Occupancy"] >= per_cu // 4


def test_workspace_size_covers_every_plan():
    rnd = random.Random(5)
    max_slots = pcr.lib()._ZN3pcr20cross_rows_max_slotsEii
    max_slots.restype, max_slots.argtypes = ctypes.c_int64, [ctypes.c_int32] * 2
    seen = set()
    for _ in range(20000):
        d, Hkv, B = rnd.choice([64, 128]), rnd.randint(1, 16), rnd.randint(1, rnd.choice([8, 300, 5000]))
        live, longest = rnd.randint(1, B), rnd.randint(1, rnd.choice([4, 40, 2000, 50000]))
        steps = rnd.randint(longest + live - 1, longest * live) * Hkv
        p = _plan(steps, B * Hkv, longest, d)
        assert 1 <= p.runs <= max(steps, B * Hkv * max(1, p.parts))
        seen.add(min(p.parts, 2))
        if p.parts == 1 or p.runs == 1:
            continue                      # no pair is cut
        assert p.slots <= min(B * Hkv * longest, max_slots(d, N_CU))
        assert p.slots == (p.runs if p.parts else 2 * p.runs)
        assert p.parts == 0 or p.runs == B * Hkv * p.parts
    assert seen == {0, 1, 2}
