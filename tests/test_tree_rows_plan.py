"""CPU: the plan that tree attention of few rows takes is the one that the tests of its forms count on."""
import ctypes
import random

import test_gpu_tree_forms as forms
import test_tree_plan as tp
from paper_2603_23049_amd import pcr


def _library(steps, pairs, longest, d, rows):
    f = pcr.lib()._ZN3pcr14tree_rows_planEllliii          # internal: pcr::tree_rows_plan
    f.restype, f.argtypes = tp.Plan, [ctypes.c_int64] * 3 + [ctypes.c_int32] * 3
    return f(steps, pairs, longest, d, rows, tp.N_CU)


def _fields(p):
    return p.runs, p.waves, p.parts, p.slots


def test_the_librarys_plan_is_the_tested_one():
    rnd = random.Random(9)
    for _ in range(20000):
        d, rows, pairs = rnd.choice([64, 128]), rnd.randint(1, 32), rnd.randint(1, rnd.choice([8, 300, 5000]))
        longest = rnd.randint(1, rnd.choice([4, 40, 2000, 50000]))
        steps = rnd.randint(longest, longest * pairs)
        assert _fields(_library(steps, pairs, longest, d, rows)) == _fields(tp._plan(steps, pairs, longest, d, rows))


def test_the_gpu_cases_reach_every_form_of_the_library(monkeypatch):
    monkeypatch.setattr(tp, "_plan", _library)
    got = {tp._form(*f) for f in forms.FORMS}
    assert len(got) == 24
