"""How a call of the attention operators is cut into workgroups, where the cache's words lie, and what the kernels need of registers.
No GPU."""
import ctypes
import os
import random
import re
import subprocess

import pytest

from paper_2203_05016_amd import build as lib_build

HERE = os.path.dirname(os.path.abspath(__file__))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
NONE = 2 ** 31 - 1       # no window
FIELDS = "decode col_tiles waves col_blocks splits split_tiles groups workspace".split()


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("plan") / "attention_plan_probe.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", lib_build.CSRC,
                           "-I", os.path.join(os.path.dirname(HERE), "include"), os.path.join(HERE, "attention_plan_probe.cpp"),
                           os.path.join(lib_build.CSRC, "attention_plan.cpp"), "-o", so])
    L = ctypes.CDLL(so)
    i, l, p = ctypes.c_int, ctypes.c_long, ctypes.c_void_p
    L.probe_cache_plan.argtypes = [i, i, i, i, l, i, l, i, i, p]
    L.probe_cache_plan.restype = None
    L.probe_prompt_plan.argtypes = [i, i, i, i, l, i, i, p]
    L.probe_prompt_plan.restype = None
    L.probe_place.argtypes = [i, i, i, i, ctypes.POINTER(i)]
    L.probe_head_bytes.restype = l
    return L


def _plan(call, *args):
    out = (ctypes.c_long * 8)()
    call(*args, out)
    return dict(zip(FIELDS, out))


def _tiles(first, last, tile, window, sinks):
    """Tiles with a key that some query at positions first to last sees"""
    low = 0 if window == NONE else max(first - window + 1, 0)
    return len({j // tile for j in list(range(min(sinks, last + 1))) + list(range(low, last + 1))})


def test_cuts_of_the_cache_cover_every_column_and_key(probe):
    rng = random.Random(5)
    parts, kernels = set(), set()
    for _ in range(3000):
        batch, heads, group = rng.choice([1, 2, 7, 64]), rng.choice([1, 2, 5, 8, 16]), rng.choice([1, 2, 4, 5, 8, 16, 71])
        D, queries = rng.choice([64, 96, 128]), rng.choice([1, 2, 5, 8, 17, 64, 500])
        length = max(int(2 ** rng.uniform(0, 13)), queries)
        window, sinks = rng.choice([(NONE, 0), (1, 0), (35, 4), (1024, 4), (300, 70)])
        tokens = batch * queries
        p = _plan(probe.probe_cache_plan, batch, heads, group, D, tokens, queries, length, window, sinks)
        assert p["decode"] if group * queries <= 64 else not p["decode"] if group * queries > 128 else True
        if p["decode"]:
            per_block = 16 * p["col_tiles"] // group * group if p["col_blocks"] > 1 else 16 * p["col_tiles"]
            assert p["col_tiles"] in (1, 2, 3, 4) and p["col_blocks"] * per_block >= group * queries
        else:
            assert p["col_blocks"] * p["waves"] >= -(-queries // 32) * group
        assert p["waves"] in (4, 8) and p["groups"] == batch * heads * p["col_blocks"] * p["splits"]
        tile = 32 if p["decode"] else 64
        # the first and the last block's queries see as many as any
        seen = max(_tiles(length - queries, length - 1, tile, window, sinks), 1)
        assert p["splits"] * p["split_tiles"] >= seen, (p, seen)
        assert p["workspace"] == (p["splits"] * heads * group * tokens * (D + 2) * 4 if p["splits"] > 1 else 0)
        # parts of a length that pays for the join, and no more workgroups than the GPU holds
        least = 4 * p["waves"] if p["decode"] else 4
        assert p["splits"] == 1 or (p["split_tiles"] >= least and p["groups"] <= 256 * 4)
        parts.add(p["splits"] > 1)
        kernels.add((p["decode"], group * queries > 64))
    assert parts == {False, True} and len(kernels) == 3


def test_cuts_of_prompts_cover_every_query(probe):
    rng = random.Random(6)
    for _ in range(1000):
        n, heads, group, D = rng.choice([1, 3, 40]), rng.choice([1, 4, 16]), rng.choice([1, 5, 8]), rng.choice([64, 96, 128])
        tokens = int(2 ** rng.uniform(0, 16))
        window, sinks = rng.choice([(NONE, 0), (1, 0), (35, 4), (2048, 4)])
        p = _plan(probe.probe_prompt_plan, n, heads, group, D, tokens, window, sinks)
        assert p["col_blocks"] * p["waves"] >= -(-tokens // 32) * group > (p["col_blocks"] - 1) * p["waves"]
        assert p["splits"] == 1 and p["workspace"] == 0 and p["groups"] == n * heads * p["col_blocks"]
        assert p["waves"] == 4 or (p["waves"] == 8 and D > 64 and p["groups"] >= 256)
        assert p["waves"] == 4 or D == 128 or min(tokens, window + sinks) >= 1536


def test_every_workgroup_has_a_place_of_its_own(probe):
    inner = ctypes.c_int()
    for batch in (1, 2, 3, 8, 9):
        for heads in (1, 2, 3, 4, 5, 8, 12, 16):
            for per_pair in (1, 3, 8, 13):
                pairs = batch * heads
                places, on = set(), [set() for _ in range(pairs)]
                for block in range(pairs * per_pair):
                    pair = probe.probe_place(block, pairs, heads, per_pair, inner)
                    places.add((pair, inner.value))
                    on[pair].add(block % 8)
                assert places == {(a, b) for a in range(pairs) for b in range(per_pair)}
                if heads % 4 == 0 and pairs % 8 == 0:
                    assert all(len(x) == 1 for x in on)
                elif heads % 4:
                    assert all(len(x) == min(8, per_pair) for x in on), (batch, heads, per_pair)


@pytest.mark.parametrize("D", [64, 96, 128])
def test_words_of_the_cache_do_not_overlap(probe, D):
    for page in (32, 64, 1024):
        for values in (0, 1):
            used = set()
            for token in range(page):
                for q in range(4):
                    at = probe.probe_code(D, token, q, values)
                    assert at % 4 == 0
                    used.update(range(at, at + D // 8, 4))
            assert used == set(range(0, page * D // 2, 4))
        assert probe.probe_head_bytes(page, D) == page * (D + 2 * (2 if D == 64 else 4))


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
def test_kernels_can_be_launched_and_do_not_spill():
    """Wavefronts per SIMD that the plan counts on; the prompts' kernel of 8 wavefronts for heads of 128 keeps what is used once per call
    in up to 80 spilled registers, those for heads of 64 in two."""
    jobs = [subprocess.Popen([HIPCC, "-x", "hip", "-c", os.path.join(lib_build.CSRC, source), "-o", os.devnull, "--offload-device-only",
                              "-Rpass-analysis=kernel-resource-usage"] + lib_build.FLAGS, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
            for source in ("launch_attention_f16.hip", "launch_attention_bf16.hip", "kv_cache.hip")]
    seen = {"decode": set(), "tile": set(), "join": set(), "write": set(), "read": set()}
    for job in jobs:
        text = job.communicate(timeout=900)[0].decode()
        assert job.returncode == 0, text[-2000:]
        for part in text.split("Function Name: ")[1:]:
            name, waves = part.split()[0], int(re.search(r"Occupancy \[waves/SIMD\]: (\d+)", part).group(1))
            spill = int(re.search(r"VGPRs Spill: (\d+)", part).group(1))
            kind = re.search(r"(decode|tile|join|write|read)_kernel", name).group(1)
            n = [int(x) for x in re.findall(r"L[ib](\d+)E", name)]
            seen[kind].add(tuple(n))
            if kind == "decode":
                _, D, tiles, wanted = n
                least = max(wanted // 4, {1: 4, 2: 3 if D < 128 else 2, 3: 2, 4: 1 if D == 128 else 2}[tiles])
                assert waves >= least and spill == 0, (name, waves, spill)
            elif kind == "tile":
                _, D, cache, wanted, tiny = n
                # workgroups of 4 for heads of 64: three of them share a CU
                assert waves >= (3 if D == 64 and wanted == 4 and not cache and not tiny else wanted // 4), (name, waves)
                assert spill <= (80 if D == 128 and not cache and wanted == 8 else 2 if D == 64 and not cache else 0), (name, spill)
            else:
                assert waves >= (4 if kind == "join" else 2) and spill == 0, (name, waves, spill)
    assert {kind: len(x) for kind, x in seen.items()} == {"decode": 46, "tile": 28, "join": 12, "write": 6, "read": 6}, seen
