"""The ways in which attention over pages divides its work: every case of division_cases.py is divided as it says."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from division_cases import CASES, lengths_and_rows

OVER = [c for c in CASES if c[0] == "line" and c[1] == 128]      # some pairs lie within one run whole

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("rules") / "libdivision.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2403_11805_amd", "csrc"),
                    os.path.join(ROOT, "tests", "attend_division_driver.cpp"), "-o", lib], check=True)
    fn = ctypes.CDLL(lib).attend_round
    fn.argtypes = [ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p] + [ctypes.c_int32] * 5 + [ctypes.c_void_p]

    def divide(lens, rows, n_kv_heads, per, max_rows, n_tokens, head_dim):
        lens, rows, run = np.asarray(lens, dtype=np.int32), np.asarray(rows, dtype=np.int32), ctypes.c_int32(0)
        r = fn(len(lens), lens.ctypes.data, rows.ctypes.data, n_kv_heads, per, max_rows, n_tokens, head_dim, ctypes.byref(run))
        return r, run.value
    return divide


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_cases_are_divided_as_they_say(rule, case):
    way, D, _, Hkv, Hq, _, N, most = case
    lens, rows = lengths_and_rows(case)
    step = 2 if D == 256 else 4
    found, run = rule(lens, rows, Hkv, Hq // Hkv, most, N, D)
    assert found == {"step": step, "two": 2 * step, "line": 1}[way]
    if way == "line":                 # some pairs are divided, and some runs go on from one pair to the next, or over one
        pairs = [[-(-n // 32) + 8] * (Hkv * -(-c * (Hq // Hkv) // 16)) for n, c in zip(lens, rows) if n and c]
        ends = np.cumsum(np.concatenate(pairs))
        assert max(p[0] for p in pairs) > run and (ends % run != 0).sum() > len(ends) // 2
        if case in OVER:
            assert (np.diff(ends // run) == 0).any()



def test_ways_meet_where_the_rule_says(rule):
    """A sequence's places are its units in whole steps: 512 workgroups take 512 of them, or of two steps, and no more."""
    for D, step in ((64, 4), (128, 4), (256, 2)):
        def way(n, units):
            return rule([32 * units] * n, [1] * n, 1, 1, 1, 32 * units, D)
        assert way(512, step) == (step, step)
        assert way(513, 2 * step) == (1, -(-513 * (2 * step + 8) // 512))
        assert way(512, 2 * step) == (2 * step, 2 * step)
        assert way(256, 2 * step) == (step, step)
