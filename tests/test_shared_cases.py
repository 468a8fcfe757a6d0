"""Which way the calls of shared_cases.py go.  No GPU."""
import ctypes
import os
import subprocess

import pytest

from paper_2203_05016_amd import build as lib_build
from shared_cases import CASES, FIELDS

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "shared_plan_probe.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", lib_build.CSRC, "-I", os.path.join(os.path.dirname(HERE), "include"),
                           os.path.join(HERE, "shared_plan_probe.cpp"), os.path.join(lib_build.CSRC, "attention_plan.cpp"), "-o", so])
    L = ctypes.CDLL(so)
    i, l, p = ctypes.c_int, ctypes.c_long, ctypes.c_void_p
    L.probe_shared_plan.argtypes = [i, l, l, i, i, i, i, l, i, l, i, p]
    L.probe_shared_plan.restype = None

    def call(**kw):
        out = (ctypes.c_long * 19)()
        L.probe_shared_plan(*(kw[n] for n in "prefixes max_sharing max_prefix batch heads group D tokens max_queries max_length keys_fit".split()), out)
        return dict(prefix=dict(zip(FIELDS, out[:8])), own=dict(zip(FIELDS, out[8:16])), behind=out[16], joins=out[17])
    return call


@pytest.mark.parametrize("case", CASES, ids=lambda c: c.name)
def test_way(plan, case):
    assert len(case.own) == len(case.counts) == sum(case.families) and len(case.prefix) == len(case.families)
    got = plan(**case.host())
    for name, want in case.plan.items():
        if isinstance(want, dict):
            assert {k: got[name][k] for k in want} == want, (name, got)
        else:
            assert got[name] == want, (name, got)
    assert case.name != "tiles, several parts" or got["own"]["splits"] > 1, got
