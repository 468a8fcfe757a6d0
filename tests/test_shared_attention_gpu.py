"""Attention of sequences that share prefixes against the definition in 64 bits, and against attention over tables that name the
prefix's pages for every sequence."""
import random

import numpy as np
import pytest
import torch

from attention_reference import attend, check, held
from gpu_util import announce
from paper_2203_05016_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN, INF = float("nan"), float("inf")
DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16}


def _tensor(rows, tokens, dtype, seed, gain=0.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, tokens, generator=g) * torch.exp(gain * torch.randn(rows, 1, generator=g))).to(dtype)


def _int(values):
    return torch.tensor(values, dtype=torch.int32).to(DEV)


class Served:
    """Prefixes, and sequences' own tokens, in one cache whose pages lie in no order and whose other slots read as NaN.  families: how
    many sequences every prefix has.  apart: the prefixes' table has room for so many pages that prefix and own tokens are attended to by kernels of their
    own, unless the host says that prefixes are short."""

    def __init__(self, prefixes, families, own, heads, D, page, dtype, seed=0, apart=False):
        self.heads, self.D, self.page, self.dtype = heads, D, page, dtype
        self.prefixes, self.own = prefixes, own
        self.family = [g for g, n in enumerate(families) for _ in range(n)]
        self.members = [sum(families[:g]) for g in range(len(families) + 1)]
        each = [-(-n // page) for n in prefixes + own]
        order = list(range(sum(each) + 2))
        random.Random(seed).shuffle(order)
        self.cache = binding.KVCache(len(order), page, heads, D, dtype, DEV)
        every = torch.arange(len(order) * page, dtype=torch.int32, device=DEV)
        junk = torch.full((heads * D, len(every)), NAN, dtype=dtype, device=DEV)
        self.cache.write(junk, junk, every)
        rows = [[order.pop() for _ in range(n)] for n in each]
        self.rows, self.k, self.v = rows, [], []
        for i, n in enumerate(prefixes + own):
            k, v = _tensor(heads * D, n, dtype, 100 * seed + 2 * i), _tensor(heads * D, n, dtype, 100 * seed + 2 * i + 1, 0)
            self.k.append(None), self.v.append(None)
            self.put(i, k, v)
        spare = (1 << 27) // (len(own) * heads * 2 * D * page) if apart else 0
        fill = lambda rows, spare=0: _int([r + [-7] * (max(len(x) for x in rows) + 1 + spare - len(r)) for r in rows])
        self.prefix_table, self.table = fill(rows[:len(prefixes)], spare), fill(rows[len(prefixes):])

    def put(self, i, k, v):
        if k.shape[1]:
            j = torch.arange(k.shape[1])
            slots = torch.tensor(self.rows[i])[j // self.page] * self.page + j % self.page
            self.cache.write(k.to(DEV), v.to(DEV), slots.int().to(DEV))
        self.k[i], self.v[i] = (torch.from_numpy(held(x)).to(self.dtype).double().numpy() for x in (k, v))

    def want(self, q, counts):
        outs, tols, at = [], [], 0
        q = q.double().cpu().numpy()
        for b, n in enumerate(counts):
            g, L = self.family[b], self.own[b]
            P = self.prefixes[g]
            k, v = (np.concatenate([x[g], x[len(self.prefixes) + b]], 1) for x in (self.k, self.v))
            for i in range(n):
                seen = P + max(0, L - n + i + 1)                  # the prefix, and own tokens up to the query's own
                o, t = attend(q[:, at + i:at + i + 1], k[:, :seen], v[:, :seen], self.D, seen - 1, self.dtype)
                outs.append(o), tols.append(t)
            at += n
        return np.concatenate(outs, 1), np.concatenate(tols, 1)

    def call(self, q, counts=None, **kw):
        if counts is not None:
            kw = dict(starts=_int([sum(counts[:b]) for b in range(len(counts) + 1)]), max_queries=max(max(counts), 1), **kw)
        if len(self.prefixes) > 1:
            kw = dict(members=_int(self.members), **kw)
        return self.cache.shared_attention(q, self.prefix_table, _int(self.prefixes), self.table, _int(self.own), **kw)


CASES = [  # prefixes, families, own, counts (None: one each), q heads, heads, D, page, dtype
    ([1], [1], [1], None, 1, 1, 64, 32, "f16"),
    ([33], [3], [1, 7, 40], None, 4, 2, 96, 32, "bf16"),
    ([64], [2], [64, 65], None, 8, 1, 128, 64, "f16"),
    ([700], [5], [30, 1, 99, 64, 31], None, 16, 2, 128, 32, "f16"),
    ([515], [17], list(range(1, 18)), None, 8, 2, 64, 64, "bf16"),
    ([2050], [9], [3] * 9, None, 40, 8, 96, 128, "f16"),
    ([100, 0, 31], [2, 3, 1], [5, 9, 1, 33, 64, 2], None, 4, 4, 64, 32, "f16"),
    ([300, 97], [3, 2], [10, 60, 3, 8, 129], [3, 1, 2, 3, 0], 10, 2, 128, 32, "bf16"),
    ([260], [4], [70, 50, 33, 32], [33, 0, 32, 5], 6, 2, 64, 32, "f16"),
    ([90], [2], [200, 150], [129, 140], 8, 2, 96, 64, "bf16"),
    ([1000], [1], [40], [40], 5, 1, 128, 32, "f16"),
    ([128, 5, 77], [1, 1, 1], [0, 3, 0], [1, 3, 2], 2, 1, 64, 32, "bf16"),
]


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[4:]) + "-%dx%d" % (max(c[0]), sum(c[1])))
def test_definition(case, apart):
    prefixes, families, own, counts, q_heads, heads, D, page, fmt = case
    announce("shared", *case, apart)
    s = Served(prefixes, families, own, heads, D, page, DTYPE[fmt], apart=apart)
    n = counts or [1] * len(own)
    q = _tensor(q_heads * D, sum(n), DTYPE[fmt], 9)
    want, tol = s.want(q, n)
    longest = max(max(own), 1), max(max(prefixes), 1)
    sharing = max(sum(n[s.members[g]:s.members[g + 1]]) for g in range(len(prefixes)))
    for kw in ({}, dict(max_length=longest[0], max_prefix=longest[1], max_sharing=max(sharing, 1))):
        got = s.call(q.to(DEV), counts, **kw)
        check(got, want, tol, case)
        assert torch.equal(got, s.call(q.to(DEV), counts, **kw))


@pytest.mark.parametrize("fmt,D,q_heads,heads,batch,prefix", [("f16", 128, 16, 2, 40, 9000), ("bf16", 64, 4, 4, 24, 20000), ("f16", 96, 8, 1, 70, 3000)])
def test_like_a_table_that_names_the_prefix(fmt, D, q_heads, heads, batch, prefix):
    """Prefixes of whole pages: attention over tables whose rows begin with the prefix's pages has the same definition."""
    announce("shared, long", fmt, D, q_heads, heads, batch, prefix)
    page, dtype = 32, DTYPE[fmt]
    prefix = prefix // page * page
    rng = random.Random(batch)
    own = [rng.randint(1, 300) for _ in range(batch)]
    each = [-(-n // page) for n in [prefix] + own]
    order = list(range(sum(each)))
    rng.shuffle(order)
    cache = binding.KVCache(sum(each), page, heads, D, dtype, DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    every = sum(each) * page
    k, v = (torch.randn(heads * D, every, generator=g, device=DEV).to(dtype) for _ in range(2))
    cache.write(k, v, torch.arange(every, dtype=torch.int32, device=DEV))
    rows = [[order.pop() for _ in range(n)] for n in each]
    fill = lambda rows: _int([r + [-1] * (max(len(x) for x in rows) - len(r)) for r in rows])
    q = torch.randn(q_heads * D, batch, generator=g, device=DEV).to(dtype)
    want = cache.attention(q, fill([rows[0] + r for r in rows[1:]]), _int([prefix + n for n in own])).double()
    got = cache.shared_attention(q, fill(rows[:1]), _int([prefix]), fill(rows[1:]), _int(own), max_length=300).double()
    # Both are off from the definition by at most the bound of attention_reference, whose terms here are, relative to the mean
    # magnitude W of the values (at most 6): scores 2 ((D + 4) 2^-24 A + 2^-22) with A below 8 D^0.5, weights half a step, sums 2 n 2^-24, the result half a step
    half = 2.0 ** -11 if fmt == "f16" else 2.0 ** -8
    off = 2 * ((D + 4) * 2.0 ** -24 * 8 * D ** 0.5 + 2.0 ** -22) + 2 * half + 2 * (prefix + 300) * 2.0 ** -24 + 2.0 ** -20
    weights = 2.0 ** -25 * (prefix + 300) * 6 if fmt == "f16" else 0
    assert (got - want).abs().max() <= 2 * (off * 6 + weights)
    assert (got - want).abs().mean() <= 2 * half * want.abs().mean() + 2.0 ** -14


@pytest.mark.parametrize("apart", [False, True])
def test_pages_that_are_not_there_and_impossible_lengths(apart):
    """They are NaN to those who see them, and to nobody else."""
    announce("shared, bad pages", apart)
    s = Served([70, 40], [2, 2], [33, 20, 40, 10], 1, 64, 32, torch.float16, apart=apart)
    q = _tensor(128, 4, torch.float16, 5)
    want, tol = s.want(q, [1] * 4)
    q = q.to(DEV)
    s.prefix_table[0, 1] = 10 ** 6
    s.table[3, 0] = -1
    bad = want.copy()
    bad[:, [0, 1, 3]] = NAN
    check(s.call(q), bad, tol, "missing pages")
    s = Served([70, 40], [2, 2], [33, 20, 40, 10], 1, 64, 32, torch.float16, apart=apart)
    s.own[2], s.prefixes[0] = 32 * s.table.shape[1] + 1, 32 * s.prefix_table.shape[1] + 1
    bad = want.copy()
    bad[:, [0, 1, 2]] = NAN
    check(s.call(q, max_length=64), bad, tol, "too long")
    # the same for many queries of a sequence
    s = Served([70, 40], [1, 1], [60, 45], 1, 64, 32, torch.float16, apart=apart)
    q, counts = _tensor(128, 65, torch.float16, 5), [25, 40]
    want, tol = s.want(q, counts)
    s.prefix_table[0, 2] = -1
    want[:, :25] = NAN
    check(s.call(q.to(DEV), counts), want, tol, "missing page, many queries")
    s.table[1, 1] = 10 ** 6
    want[:, 25 + 32 - 5:] = NAN                                     # own positions 32 and up
    check(s.call(q.to(DEV), counts), want, tol, "missing own page, many queries")


@pytest.mark.parametrize("apart", [False, True])
def test_nothing_to_see_and_infinities(apart):
    announce("shared, empty", apart)
    s = Served([0, 50], [2, 1], [0, 4, 0], 2, 64, 32, torch.bfloat16, apart=apart)
    q = _tensor(256, 3, torch.bfloat16, 6)
    want, tol = s.want(q, [1, 1, 1])
    assert (want[:, 0] == 0).all() and (want[:, 1:] != 0).any()
    check(s.call(q.to(DEV)), want, tol, "empty")
    # a block of values that is not finite, in the prefix of one family, is that family's
    s = Served([40, 50], [1, 2], [3, 4, 5], 2, 64, 32, torch.bfloat16, apart=apart)
    k, v = _tensor(128, 50, torch.bfloat16, 7), _tensor(128, 50, torch.bfloat16, 8)
    v[70, 49] = INF
    s.put(1, k, v)
    want, tol = s.want(q, [1, 1, 1])
    got = s.call(q.to(DEV))
    assert np.isnan(want[128:, 1:]).any() and not np.isnan(want[:, 0]).any()
    check(got, want, tol, "infinity")


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("counts", [None, [2, 1, 3], [9, 0, 12], [20, 31, 33]])
def test_columns_of_no_sequence_stay(counts, apart):
    """Columns before the first sequence's and behind the last one's, and what lies around the result."""
    announce("shared, columns", counts, apart)
    dtype = torch.float16
    s = Served([3000], [3], [20, 30, 40], 2, 64, 32, dtype, apart=apart)
    n = counts or [1, 1, 1]
    q = _tensor(256, sum(n), dtype, 5)
    want, tol = s.want(q, n)
    check(s.call(q.to(DEV), counts), want, tol, "as it is")
    wide = torch.full((256, sum(n) + 9), 3.0, dtype=dtype, device=DEV)
    wide[:, 4:4 + sum(n)] = q.to(DEV)
    starts = _int([4 + sum(n[:b]) for b in range(4)])
    memory = torch.full((256, sum(n) + 15), 5.0, dtype=dtype, device=DEV)
    out = memory[:, 3:-3]
    got = s.cache.shared_attention(wide, s.prefix_table, _int(s.prefixes), s.table, _int(s.own), starts=starts, max_queries=max(n), out=out)
    assert got is out
    check(out[:, 4:4 + sum(n)], want, tol, "among others")          # (other bounds may cut the work otherwise)
    assert (memory[:, :7] == 5).all() and (memory[:, 7 + sum(n):] == 5).all()


def test_bounds_of_the_host_that_are_too_small_or_too_large():
    """max_length and max_prefix decide how the work is cut only; larger max_queries and max_sharing change nothing."""
    announce("shared, bounds")
    s = Served([3000], [3], [700, 30, 1], 1, 128, 32, torch.float16, apart=True)
    q = _tensor(512, 3, torch.float16, 5)
    want, tol = s.want(q, [1, 1, 1])
    for kw in (dict(max_length=1, max_prefix=1), dict(max_length=32 * s.table.shape[1], max_prefix=32 * s.prefix_table.shape[1], max_sharing=2 ** 31 - 1)):
        check(s.call(q.to(DEV), **kw), want, tol, kw)
    check(s.call(q.to(DEV), [1, 1, 1], max_sharing=1000), want, tol, "starts")


@pytest.mark.parametrize("max_prefix", [500, None])
def test_graphs_and_streams(max_prefix):
    """Two captured calls that share the allocator's pool, replayed in turn while lengths grow; and another stream."""
    announce("shared, graphs", max_prefix)
    dtype = torch.float16
    s = Served([500], [4], [100, 20, 60, 90], 2, 64, 32, dtype, apart=True)
    prefix, own = _int([500]), _int([1, 1, 1, 1])
    qs = [_tensor(512, 4, dtype, 20 + i).to(DEV) for i in range(2)]
    call = lambda q, **kw: s.cache.shared_attention(q, s.prefix_table, prefix, s.table, own, max_length=100, max_prefix=max_prefix, **kw)
    for q in qs:
        call(q)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for q in qs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], pool=graphs[0].pool() if len(graphs) > 1 else None):
            outs.append(call(q))
    for step in range(3):
        own.copy_(_int([100 - step, 1 + step, 60, 33 * step]))
        for graph, out, q in zip(graphs, outs, qs):
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, call(q))
    side = torch.cuda.Stream()
    want = call(qs[0])
    torch.cuda.synchronize()
    got = call(qs[0], stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_kernels_that_run():
    """Few sequences behind short prefixes, many, and prompts: the kernels that run, and that they agree where the host's bounds choose between them."""
    announce("shared, kernels")
    name = lambda: binding.last_kernel()
    s = Served([200], [70], [5] * 70, 1, 64, 32, torch.float16, apart=True)
    q = _tensor(256, 70, torch.float16, 1)
    want, tol = s.want(q, [1] * 70)
    check(s.call(q.to(DEV), max_prefix=200, max_length=5), want, tol, "together")
    assert name().startswith("shflbw_attention_decode_kernel<64,16 columns")
    check(s.call(q.to(DEV), max_length=5), want, tol, "apart")
    assert name().startswith("shflbw_attention_tile_kernel<64,cache")      # 280 columns of the prefix
    s = Served([200], [20], [5] * 20, 1, 64, 32, torch.float16, apart=True)
    s.call(_tensor(64, 20, torch.float16, 1).to(DEV))
    assert name().startswith("shflbw_attention_decode_kernel<64,32 columns")
    s = Served([200], [2], [30] * 2, 1, 64, 32, torch.float16)
    s.call(_tensor(64, 40, torch.float16, 1).to(DEV), [20, 20])
    assert name().startswith("shflbw_attention_tile_kernel<64,cache")
