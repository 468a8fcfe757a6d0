"""The attention operators at the limits of what a call may ask for.  No GPU."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2203_05016_amd import binding, build as lib_build

HERE = os.path.dirname(os.path.abspath(__file__))
NONE = 2 ** 31 - 1       # no window


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("limits") / "attention_limits_probe.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", lib_build.CSRC,
                           "-I", os.path.join(os.path.dirname(HERE), "include"), os.path.join(HERE, "attention_limits_probe.cpp"),
                           os.path.join(lib_build.CSRC, "attention_plan.cpp"), "-o", so])
    L = ctypes.CDLL(so)
    i, l = ctypes.c_int, ctypes.c_long
    L.probe_prompt_kernel.argtypes = [i, i, i, i, l, i, i, l, ctypes.POINTER(i)]
    L.probe_cache_blocks.argtypes = [i, i, i, i, l, i, l, ctypes.POINTER(l)]
    L.probe_cache_blocks.restype = None
    return L


def test_the_kernel_that_is_launched_covers_every_query_of_a_prompt(probe):
    """All column counts around one tile of keys, many sequences and heads: the kernel named exists, is the form for fewer than 64
    columns exactly there, and its workgroups have an item for every block of queries of every head."""
    out = (ctypes.c_int * 3)()
    named = set()
    for tokens in list(range(1, 67)) + [100, 5000]:
        for sequences in (1, 2, 16, 20, 32, 64, 300):
            for heads in (1, 4, 8, 16, 32):
                for group in (1, 5, 8, 16):
                    for D in (64, 96, 128):
                        for most in {1, -(-tokens // sequences), tokens}:
                            for window, sinks in ((NONE, 0), (16, 2)):
                                assert probe.probe_prompt_kernel(sequences, heads, group, D, most, window, sinks, tokens, out)
                                waves, tiny, blocks = out
                                assert tiny == (tokens < 64) and (waves == 4 or not tiny)
                                assert blocks * waves >= -(-most // 32) * group, (tokens, sequences, heads, group, D, most)
                                named.add((D, waves, tiny))
    assert named == {(64, 4, 0), (96, 4, 0), (96, 8, 0), (128, 4, 0), (128, 8, 0), (64, 4, 1), (96, 4, 1), (128, 4, 1)}


def test_a_generous_bound_of_queries_cuts_as_the_columns_do(probe):
    """No sequence has more queries than there are columns in all."""
    one, two = (ctypes.c_long * 3)(), (ctypes.c_long * 3)()
    for batch in (1, 3, 64):
        for group in (1, 8, 33, 65535):
            for D in (64, 128):
                for tokens in (1, 7, 64, 1000):
                    probe.probe_cache_blocks(batch, 2, group, D, tokens, tokens, 5000, one)
                    for most in (tokens + 1, 100000, 2 ** 31 - 1):
                        probe.probe_cache_blocks(batch, 2, group, D, tokens, most, 5000, two)
                        assert list(one) == list(two) and one[0] > 0 and one[1] > 0, (batch, group, D, tokens, most, list(two))


def test_more_workgroups_than_a_launch_takes_are_counted_as_such(probe):
    """Never as few, or fewer than none: the launcher refuses by this number."""
    out = (ctypes.c_long * 3)()
    for batch, heads, group, tokens in ((1, 1, 65535, 2 ** 31 - 1), (2 ** 31 - 1, 16384, 3, 2 ** 31 - 1), (1000, 16384, 4, 2 ** 31 - 1)):
        probe.probe_cache_blocks(batch, heads, group, 128, tokens, 2 ** 31 - 1, 5000, out)
        assert out[1] > 2 ** 31 - 1 and out[0] > 0, list(out)


@pytest.mark.parametrize("pages,page,heads,D", [(1, 32, 16384, 128), (1, 32, 16385, 64), (1, 32, 20000, 96), (1 << 21, 1024, 1, 64), (1 << 26, 32, 1, 64)])
def test_caches_that_no_call_takes_have_no_size(pages, page, heads, D):
    """shflbw_kv_cache_bytes gives 0 for what the calls refuse, before memory is laid out for it, and the calls say why."""
    L = binding.lib()
    assert L.shflbw_kv_cache_bytes(pages, page, heads, D) == 0
    cache = binding._Cache(128, pages, page, heads, D, binding.F16)
    assert L.shflbw_kv_write(cache, 1, 9, 1, 9, 1, 9, None) == -2 and ("heads" if heads > 1 else "slots") in binding.last_error()
    with pytest.raises(ValueError, match="heads" if heads > 1 else "slots"):
        binding.KVCache(pages, page, heads, D, torch.float16)


def test_the_largest_caches_have_one():
    size = binding.lib().shflbw_kv_cache_bytes
    assert size(1, 32, 16384, 64) == 16384 * 32 * 68 and size(1, 32, 16383, 128) == 16383 * 32 * 136
    assert size((1 << 21) - 1, 1024, 1, 64) == ((1 << 21) - 1) * 1024 * 68
