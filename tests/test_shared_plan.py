"""How attention over shared prefixes is cut into workgroups, and what the kernels around a shared cache need of registers.  No GPU."""
import ctypes
import os
import random
import re
import subprocess

import pytest

from paper_2203_05016_amd import build as lib_build

HERE = os.path.dirname(os.path.abspath(__file__))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FIELDS = "decode col_tiles waves col_blocks splits split_tiles groups tiny".split()


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "shared_plan_probe.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", lib_build.CSRC,
                           "-I", os.path.join(os.path.dirname(HERE), "include"), os.path.join(HERE, "shared_plan_probe.cpp"),
                           os.path.join(lib_build.CSRC, "attention_plan.cpp"), "-o", so])
    L = ctypes.CDLL(so)
    i, l, p = ctypes.c_int, ctypes.c_long, ctypes.c_void_p
    L.probe_shared_plan.argtypes = [i, l, l, i, i, i, i, l, i, l, i, p]
    L.probe_shared_plan.restype = None

    def call(**kw):
        out = (ctypes.c_long * 19)()
        L.probe_shared_plan(*(kw[n] for n in "prefixes max_sharing max_prefix batch heads group D tokens max_queries max_length keys_fit".split()), out)
        return dict(prefix=dict(zip(FIELDS, out[:8])), own=dict(zip(FIELDS, out[8:16])), behind=out[16], joins=out[17], workspace=out[18])
    call.joined = L.probe_most_joined()
    return call


def _covers(p, pairs, group, queries, keys, flat):
    """Every column has a workgroup, every tile of keys a part."""
    assert p["waves"] in (4, 8) and not p["tiny"] and p["splits"] >= 1
    if p["decode"]:
        assert p["col_tiles"] in (1, 2, 3, 4)
        columns = 16 * p["col_tiles"]
        assert p["col_blocks"] == 1 or columns // group > 0
        assert p["col_blocks"] * (columns // group * group if p["col_blocks"] > 1 else columns) >= group * queries
    else:
        items = -(-group * queries // 32) if flat else -(-queries // 32) * group
        assert p["col_blocks"] * p["waves"] >= items
    assert p["splits"] * p["split_tiles"] * (32 if p["decode"] else 64) >= keys
    assert p["groups"] == pairs * p["col_blocks"] * p["splits"]


def test_cuts_cover_every_column_and_key(plan):
    rng, kinds = random.Random(7), set()
    for _ in range(4000):
        prefixes, each = rng.choice([1, 1, 2, 16]), int(2 ** rng.uniform(0, 7))
        heads, group, D = rng.choice([1, 2, 8, 16]), rng.choice([1, 2, 4, 5, 8, 33, 71]), rng.choice([64, 96, 128])
        queries, length, prefix = rng.choice([1, 1, 2, 5, 9, 19, 20, 64, 500]), int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 17))
        batch, fit = prefixes * each, rng.random() < 0.9
        p = plan(prefixes=prefixes, max_sharing=each * queries, max_prefix=prefix, batch=batch, heads=heads, group=group, D=D, tokens=batch * queries,
                 max_queries=queries, max_length=length, keys_fit=fit)
        rows = 4 * (D + 2) * heads * group * batch * queries
        kinds.add((p["behind"], p["joins"], p["own"]["decode"], p["prefix"]["decode"]))
        if p["behind"]:
            assert fit and not p["joins"]
            _covers(p["own"], batch * heads, group, queries, prefix + length, False)
            assert p["workspace"] == (p["own"]["splits"] > 1) * p["own"]["splits"] * rows
            continue
        _covers(p["own"], batch * heads, group, queries, length, False)
        _covers(p["prefix"], prefixes * heads, group, each * queries, prefix, True)
        if p["joins"]:
            assert p["own"]["decode"] and p["own"]["splits"] == 1 and p["prefix"]["splits"] <= plan.joined
        assert p["workspace"] == (p["prefix"]["splits"] + (0 if p["joins"] else p["own"]["splits"])) * rows
    assert kinds >= {(1, 0, 1, 0), (1, 0, 0, 0), (0, 1, 1, 1), (0, 1, 1, 0), (0, 0, 1, 1), (0, 0, 0, 0)}, kinds


def test_bounds_past_the_columns_and_counts_past_32_bits(plan):
    base = dict(prefixes=1, max_sharing=2 ** 40, max_prefix=10 ** 6, batch=64, heads=8, group=8, D=128, tokens=64, max_queries=2 ** 31 - 1, max_length=300, keys_fit=0)
    p, q = plan(**base), plan(**{**base, "max_sharing": 64, "max_queries": 64})
    assert p == q
    p = plan(**{**base, "tokens": 2 ** 31 - 1, "batch": 2 ** 31 - 1, "max_queries": 1, "group": 8191, "heads": 8})
    assert p["workspace"] > 2 ** 50 and p["prefix"]["groups"] > 2 ** 31 - 1


def test_kernels_can_be_launched_and_do_not_spill():
    """Wavefronts per SIMD that the launchers count on: those of attention with prefixes are as those without.  Blocks of 32 columns of heads of 96 keep four
    values that are used once per call in spilled registers."""
    jobs = [subprocess.Popen([HIPCC, "-x", "hip", "-c", os.path.join(lib_build.CSRC, source), "-o", os.devnull, "--offload-device-only",
                              "-Rpass-analysis=kernel-resource-usage"] + lib_build.FLAGS, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
            for source in ("launch_shared_attention_f16.hip", "launch_shared_attention_bf16.hip", "kv_pages.hip", "norm_rotate.hip")]
    seen = {}
    for job in jobs:
        text = job.communicate(timeout=900)[0].decode()
        assert job.returncode == 0, text[-2000:]
        for part in text.split("Function Name: ")[1:]:
            name, waves = part.split()[0], int(re.search(r"Occupancy \[waves/SIMD\]: (\d+)", part).group(1))
            spill, lds = (int(re.search(r"%s: (\d+)" % x, part).group(1)) for x in ("VGPRs Spill", r"LDS Size \[bytes/block\]"))
            kind = re.search(r"\d([a-z_]+)_kernel", name).group(1)
            n = [int(x) for x in re.findall(r"L[ib](\d+)E", name)]
            seen.setdefault(kind, set()).add(tuple(n))
            assert spill <= (4 if kind == "attention_decode" and n[1:3] == [96, 2] else 0) and lds <= 160 * 1024, (name, spill, lds)
            if kind == "attention_decode":
                _, D, tiles, wanted = n
                assert waves >= max(wanted // 4, {1: 4, 2: 3 if D < 128 else 2, 3: 2, 4: 1 if D == 128 else 2}[tiles]), (name, waves)
            elif kind == "attention_tile":
                assert waves >= n[3] // 4, (name, waves)
            elif kind.startswith("norm_rotate"):
                assert waves >= 2, (name, waves)
            else:
                assert waves >= 4, (name, waves)      # workgroups of 1024
    assert {k: len(x) for k, x in seen.items() if "attention" in k or "rotate" in k} == {
        "attention_decode": 46, "attention_tile": 12, "attention_join": 12, "norm_rotate": 18, "norm_rotate_few": 12}, seen
