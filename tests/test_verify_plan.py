"""CPU: how verification is cut up: that the GPU tests' cases take every number of rounds, with walks that end in each of
them and after the last, workgroups whose waves sum several tiles, and tiles of several pieces; and that no
plan needs more workspace than the size query says."""
import ctypes
import random

import pytest

import test_gpu_verify_rounds as rounds
from paper_2603_23049_amd import pcr


class Plan(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in ("tiles", "pieces", "rounds", "wgs")] + [("bytes", ctypes.c_int64)]


def _plan(B, T, V, drawn):
    f = pcr.lib()._ZN3pcr11verify_planEiiib          # internal: pcr::verify_plan
    f.restype, f.argtypes = Plan, [ctypes.c_int32] * 3 + [ctypes.c_bool]
    return f(B, T, V, drawn)


def _of(name):
    n, V, drawn, _, _ = rounds.CASES[name]
    return _plan(len(n), sum(n), V, drawn)


def test_cases_take_every_form():
    p = {name: _of(name) for name in rounds.CASES}
    assert {x.rounds for x in p.values()} == {1, 2, 4}                  # (none: the short vocabularies of test_gpu_verify)
    assert _plan(4, 40, 8192, True).rounds == 0
    for name, x in p.items():
        want = 4 if "four" in name else 2 if "two rounds" in name else 1
        assert x.rounds == want and x.pieces == (2 if "pieces" in name else 1), name
    for name in ("four rounds, many sequences", "one round, many sequences", "one round, no probabilities, many sequences"):
        assert p[name].wgs * 4 < p[name].tiles                          # several tiles a wave


@pytest.mark.parametrize("name,least", [("four rounds", {1, 2, 3, 4}), ("four rounds, bushes", {5}),
                                        ("four rounds, many sequences", {1, 2, 3, 4, 5}), ("two rounds", {1, 3}),
                                        ("two rounds, more sequences", {1, 2, 3})])
def test_walks_end_in_every_round(name, least):
    got = rounds.passes(rounds.case(name))
    assert least <= {min(x, 5) for x in got}, got


def test_workspace_size_covers_every_plan():
    rnd, n = random.Random(7), ctypes.c_int64(0)
    for _ in range(3000):
        V, B = rnd.choice([1, 8192, 8193, 50000, 128000, 4194304, 4194305, 2 ** 30]), rnd.randint(1, rnd.choice([8, 300, 5000]))
        T = rnd.randint(B, 20 * B)
        assert pcr.lib().pcr_verify_drafts_workspace_size(B, T, V, ctypes.byref(n)) == 0
        for _ in range(4):
            b = rnd.randint(1, B)
            p = _plan(b, rnd.randint(0, T), V, rnd.random() < 0.5)
            assert p.bytes <= n.value and (p.bytes > 0) == (p.rounds > 0)
            assert p.tiles <= 4096 and p.tiles * p.pieces * 1024 >= V and p.wgs >= 1
