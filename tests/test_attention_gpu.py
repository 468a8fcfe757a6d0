"""Attention over the 4-bit cache and windowed attention of prompts against their definition in 64 bits, at the lengths,
masks, layouts and values where they can go wrong."""
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


def _tensor(rows, tokens, dtype, seed, gain=0.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, tokens, generator=g) * torch.exp(gain * torch.randn(rows, 1, generator=g))).to(dtype)


class Served:
    """Sequences of the given lengths in a cache, whose pages lie in no order; `spoil` fills every slot that no sequence has with
    blocks that read as NaN."""

    def __init__(self, lengths, heads, D, page, dtype, seed=0, spoil=True, spare=1):
        self.heads, self.D, self.page, self.dtype, self.lengths = heads, D, page, dtype, lengths
        each = [-(-n // page) for n in lengths]
        width = max(max(each), 1) + spare
        pages = sum(each) + 2
        order = list(range(pages))
        random.Random(seed).shuffle(order)
        self.table = torch.full((len(lengths), width), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(each):
            self.table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        self.cache = binding.KVCache(pages, page, heads, D, dtype, DEV)
        if spoil:
            every = torch.arange(pages * page, dtype=torch.int32, device=DEV)
            junk = torch.full((heads * D, pages * page), NAN, dtype=dtype, device=DEV)
            self.cache.write(junk, junk, every)
        self.k, self.v = [], []
        for b, n in enumerate(lengths):
            k, v = _tensor(heads * D, n, dtype, 100 * seed + 2 * b), _tensor(heads * D, n, dtype, 100 * seed + 2 * b + 1, 0)
            self.put(b, k, v)

    def slots(self, b, n):
        j = torch.arange(n)
        return (self.table[b].long()[j // self.page] * self.page + j % self.page).int()

    def put(self, b, k, v):
        if k.shape[1]:
            self.cache.write(k.to(DEV), v.to(DEV), self.slots(b, k.shape[1]).to(DEV))
        kd, vd = (torch.from_numpy(held(x)).to(self.dtype).double().numpy() for x in (k, v))
        self.k[b:b + 1], self.v[b:b + 1] = [kd], [vd]

    def want(self, q, counts, **mask):
        outs, tols, at = [], [], 0
        for b, (n, nq) in enumerate(zip(self.lengths, counts)):
            o, t = attend(q[:, at:at + nq].double().numpy(), self.k[b], self.v[b], self.D, n - nq, self.dtype, **mask)
            outs.append(o)
            tols.append(t)
            at += nq
        return np.concatenate(outs, 1), np.concatenate(tols, 1)

    def run(self, q, counts=None, **kw):
        starts, most = None, 1
        if counts is not None:
            starts = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device=DEV)
            most = max(max(counts), 1)
        kw.setdefault("max_length", max(max(self.lengths), 1))
        return self.cache.attention(q.to(DEV) if q.device.type == "cpu" else q, self.table.to(DEV),
                                    torch.tensor(self.lengths, dtype=torch.int32, device=DEV), starts=starts, max_queries=most, **kw)


MASKS = [(0, 0), (1, 0), (1, 3), (40, 4), (33, 40), (64, 0), (4096, 5)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D,heads,group,page", [(64, 2, 1, 32), (96, 1, 5, 64), (128, 2, 8, 128), (64, 1, 17, 64), (128, 1, 33, 32), (96, 1, 64, 32)])
def test_one_token_each(dtype, D, heads, group, page):
    lengths = [1, 0, 31, 32, 33, 64, 65, 200, 7]
    s = Served(lengths, heads, D, page, dtype, seed=1)
    q = _tensor(heads * group * D, len(lengths), dtype, 50)
    for window, sinks in MASKS:
        announce("decode", dtype, D, heads, group, page, window, sinks)
        got = s.run(q, window=window, sinks=sinks)
        assert "decode_kernel<%d,%d columns" % (D, (group + 15) // 16 * 16) in binding.last_kernel()
        check(got, *s.want(q, [1] * len(lengths), window=window, sinks=sinks), "window %d sinks %d" % (window, sinks))
        assert not got[:, 1].any()                               # a sequence of no tokens sees nothing


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D,heads,group,page", [(64, 2, 2, 32), (96, 1, 5, 64), (128, 2, 8, 32)])
def test_some_tokens_each(dtype, D, heads, group, page):
    lengths, counts = [5, 3, 34, 97, 128, 0, 260, 6], [5, 5, 2, 5, 1, 2, 4, 0]   # more queries than tokens, and none
    s = Served(lengths, heads, D, page, dtype, seed=2)
    q = _tensor(heads * group * D, sum(counts), dtype, 51)
    for window, sinks in MASKS:
        announce("draft", dtype, D, heads, group, page, window, sinks)
        got = s.run(q, counts, window=window, sinks=sinks)
        assert "decode_kernel" in binding.last_kernel()
        check(got, *s.want(q, counts, window=window, sinks=sinks), "window %d sinks %d" % (window, sinks))
        assert not got[:, 5:7].any()                             # positions -2 and -1


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D,heads,group,page", [(64, 2, 1, 32), (96, 1, 5, 64), (128, 1, 8, 128)])
def test_many_tokens_each(dtype, D, heads, group, page):
    lengths, counts = [70, 130, 300, 65, 20, 129], [70, 33, 100, 1, 25, 0]
    s = Served(lengths, heads, D, page, dtype, seed=3)
    q = _tensor(heads * group * D, sum(counts), dtype, 52)
    for window, sinks in MASKS:
        announce("chunk", dtype, D, heads, group, page, window, sinks)
        got = s.run(q, counts, window=window, sinks=sinks)
        assert ("decode_kernel<%d,32 columns" if group == 1 else "tile_kernel<%d,cache") % D in binding.last_kernel()
        check(got, *s.want(q, counts, window=window, sinks=sinks), "window %d sinks %d" % (window, sinks))


@pytest.mark.parametrize("D", [64, 96, 128])
def test_more_tokens_of_single_heads(D):
    lengths, counts = [200, 3, 300], [140, 3, 129]
    s = Served(lengths, 2, D, 32, torch.float16, seed=23)
    q = _tensor(2 * D, sum(counts), torch.float16, 54)
    for window, sinks in MASKS:
        announce("more tokens", D, window, sinks)
        got = s.run(q, counts, window=window, sinks=sinks)
        assert "tile_kernel<%d,cache" % D in binding.last_kernel()
        check(got, *s.want(q, counts, window=window, sinks=sinks), "window %d sinks %d" % (window, sinks))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D,heads,group", [(64, 2, 1), (96, 1, 5), (128, 1, 8)])
@pytest.mark.parametrize("lengths", [[1], [77], [64, 1, 0, 130, 33], [8, 300], [31, 32, 257]])
def test_prompts(dtype, D, heads, group, lengths):
    tokens = sum(lengths)
    q, k, v = (_tensor(n * D, tokens, dtype, 60 + i, 0.5 if i < 2 else 0) for i, n in enumerate((heads * group, heads, heads)))
    starts = torch.tensor([0] + list(np.cumsum(lengths)), dtype=torch.int32, device=DEV)
    for window, sinks in MASKS:
        announce("prompt", dtype, D, heads, group, lengths, window, sinks)
        got = binding.window_attention(q.to(DEV), k.to(DEV), v.to(DEV), D, starts, max(lengths), window, sinks)
        assert "tile_kernel<%d,prompt" % D in binding.last_kernel()
        at = 0
        for n in lengths:
            part = [x[:, at:at + n].double().numpy() for x in (q, k, v)]
            check(got[:, at:at + n], *attend(*part, D, 0, dtype, window=window, sinks=sinks), "window %d sinks %d" % (window, sinks))
            at += n
    if len(lengths) == 1:
        assert torch.equal(got, binding.window_attention(q.to(DEV), k.to(DEV), v.to(DEV), D, window=window, sinks=sinks))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("counts", [None, [3, 5], [80, 41]])
@pytest.mark.parametrize("D,group", [(64, 2), (128, 8)])
def test_long_contexts_are_split(dtype, counts, D, group):
    announce("split", dtype, counts, D, group)
    lengths = [2500, 1111]
    s = Served(lengths, 1, D, 64, dtype, seed=4)
    q = _tensor(group * D, sum(counts) if counts else 2, dtype, 53)
    seqs = binding._Sequences(group, 2, max(counts or [1]), s.table.shape[1], 0, 0, q.shape[1], 2500, s.table.shape[1], None, None, 1 if counts else None)
    assert binding.lib().shflbw_kv_attention_workspace(s.cache._c, seqs) > 0
    for window, sinks in [(0, 0), (900, 70)]:
        got = s.run(q, counts, window=window, sinks=sinks)
        check(got, *s.want(q, counts or [1, 1], window=window, sinks=sinks), "window %d" % window)
        assert torch.equal(got, s.run(q, counts, window=window, sinks=sinks))       # the same bits again
        check(s.run(q, counts, window=window, sinks=sinks, max_length=None), *s.want(q, counts or [1, 1], window=window, sinks=sinks))


@pytest.mark.parametrize("counts", [None, [4, 3], [70, 40]])
def test_values_that_are_not_finite(counts):
    """Hidden ones leave a query alone, seen ones reach it: blocks of the cache that read as NaN at keys only later queries
    see, at keys that only the window of earlier ones holds, and at seen ones."""
    dtype, D, group = torch.bfloat16, 64, 2
    lengths = [150, 75]
    q = _tensor(2 * group * D, sum(counts) if counts else 2, dtype, 54)
    for places in ([149], [148, 74], [60], [100, 3], [0]):
        announce("not finite", counts, places)
        s = Served(lengths, 2, D, 32, dtype, seed=5)
        for b, n in enumerate(lengths):
            k, v = _tensor(2 * D, n, dtype, 7 + b), _tensor(2 * D, n, dtype, 9 + b, 0)
            for j in places:
                if j < n:
                    v[40, j] = INF                              # features 32..63 of head 0 of that token
                    if j == 3:
                        k[70, j] = NAN                          # a key of head 1
            s.put(b, k, v)
        for window, sinks in [(0, 0), (30, 0), (20, 2), (45, 10)]:
            got = s.run(q, counts, window=window, sinks=sinks)
            check(got, *s.want(q, counts or [1, 1], window=window, sinks=sinks), "%r window %d sinks %d" % (places, window, sinks))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_prompt_values_that_are_not_finite(dtype):
    D, lengths = 64, [90, 45]
    starts = torch.tensor([0, 90, 135], dtype=torch.int32, device=DEV)
    for place, bad in ((89, NAN), (90, INF), (20, -INF), (0, NAN), (70, INF), (134, NAN)):
        q, k, v = (_tensor(2 * D, 135, dtype, 70 + i, 0.3) for i in range(3))
        v[5, place], v[100, place] = bad, bad
        k[80, place] = NAN                                       # the keys of head 1 as well
        for window, sinks in [(0, 0), (16, 0), (16, 2)]:
            announce("prompt not finite", dtype, place, bad, window, sinks)
            got = binding.window_attention(q.to(DEV), k.to(DEV), v.to(DEV), D, starts, 90, window, sinks)
            for at, n in ((0, 90), (90, 45)):
                part = [x[:, at:at + n].double().numpy() for x in (q, k, v)]
                check(got[:, at:at + n], *attend(*part, D, 0, dtype, window=window, sinks=sinks), "%d window %d" % (place, window))


@pytest.mark.parametrize("counts", [None, [4, 3], [9, 6], [24, 30], [70, 40]])
def test_the_same_bits_again(counts):
    """Ten calls with the same arguments, masked and not: what a wait state or a barrier left out would show."""
    for dtype, D in ((torch.float16, 64), (torch.bfloat16, 128)):
        announce("the same bits", counts, dtype, D)
        s = Served([1200, 700], 2, D, 64, dtype, seed=11)
        q = _tensor(4 * D, sum(counts) if counts else 2, dtype, 59)
        for mask in (dict(), dict(window=300, sinks=3)):
            first = s.run(q, counts, **mask)
            for _ in range(10):
                assert torch.equal(first, s.run(q, counts, **mask))
    prompt = [_tensor(4 * 64, 500, torch.float16, 61 + i, 0.3).to(DEV) for i in range(3)]
    first = binding.window_attention(*prompt, 64, window=100, sinks=5)
    for _ in range(10):
        assert torch.equal(first, binding.window_attention(*prompt, 64, window=100, sinks=5))


def test_large_and_small_scores():
    """Scores whose exponentials leave 32 bits, all equal scores, and rows of zeros."""
    dtype, D, n = torch.float16, 64, 100
    for gain in (0.0, 1e-3, 30.0, 1000.0):
        announce("scores", gain)
        q, k, v = (_tensor(D, n, dtype, 80 + i, 0) for i in range(3))
        q = (q * gain).to(dtype)
        got = binding.window_attention(q.to(DEV), k.to(DEV), v.to(DEV), D)
        check(got, *attend(q.double().numpy(), k.double().numpy(), v.double().numpy(), D, 0, dtype), "gain %g" % gain)
        s = Served([n], 1, D, 32, dtype, seed=6)
        check(s.run(q[:, -1:]), *s.want(q[:, -1:], [1]), "cache, gain %g" % gain)


def test_strides_and_odd_rows():
    announce("strides")
    dtype, D, lengths = torch.float16, 96, [50, 81]
    tokens = sum(lengths)
    starts = torch.tensor([0, 50, 131], dtype=torch.int32, device=DEV)
    bufs = [torch.full((rows * D, ld), NAN, dtype=dtype, device=DEV) for rows, ld in ((4, 177), (2, 140), (2, 151), (4, 163))]
    q, k, v, out = (x[:, at:at + tokens] for x, at in zip(bufs, (3, 9, 1, 5)))
    for i, x in enumerate((q, k, v)):
        x.copy_(_tensor(x.shape[0], tokens, dtype, 90 + i, 0.3))
    assert binding.window_attention(q, k, v, D, starts, 81, 40, 3, out=out) is out
    at = 0
    for n in lengths:
        check(out[:, at:at + n], *attend(*[x[:, at:at + n].double().cpu().numpy() for x in (q, k, v)], D, 0, dtype, window=40, sinks=3))
        at += n
    assert torch.isnan(bufs[3][:, :5]).all() and torch.isnan(bufs[3][:, 5 + tokens:]).all()
    s = Served([40, 90], 2, D, 32, dtype, seed=7)
    for counts in (None, [3, 2], [40, 60]):
        n = sum(counts) if counts else 2
        wide, res = torch.full((4 * D, n + 7), NAN, dtype=dtype, device=DEV), torch.full((4 * D, n + 4), NAN, dtype=dtype, device=DEV)
        wide[:, 5:5 + n] = _tensor(4 * D, n, dtype, 95)
        s.run(wide[:, 5:5 + n], counts, out=res[:, 1:1 + n])
        check(res[:, 1:1 + n], *s.want(wide[:, 5:5 + n].cpu(), counts or [1, 1]))
        assert torch.isnan(res[:, 0]).all() and torch.isnan(res[:, 1 + n:]).all()


@pytest.mark.parametrize("counts", [None, [2, 3, 1], [70, 10, 40]])
def test_pages_that_are_not_there(counts):
    """A page outside the cache reads as NaN, and only for those who see it; a length beyond the table's pages is NaN."""
    announce("bad pages", counts)
    dtype, D = torch.float16, 64
    lengths = [100, 80, 120]
    s = Served(lengths, 1, D, 32, dtype, seed=8, spare=0)
    n = counts or [1, 1, 1]
    q = _tensor(2 * D, sum(n), dtype, 55)
    want, tol = s.want(q, n)
    good = s.table.clone()
    for bad in (-1, s.cache.pages, 2 ** 31 - 1, -2 ** 31):
        s.table = good.clone()
        s.table[1, 1] = bad                                      # tokens 32..63 of sequence 1
        w = want.copy()
        w[:, n[0]:n[0] + n[1]] = NAN
        check(s.run(q, counts), w, tol, "page %d" % bad)
        w = want.copy()
        part, t = attend(q[:, n[0]:n[0] + n[1]].double().numpy(), s.k[1], s.v[1], D, 80 - n[1], dtype, window=5)
        got = s.run(q, counts, window=5)
        check(got[:, n[0]:n[0] + n[1]], part, t, "page %d outside the window" % bad)
    s.table = good
    s.lengths = [100, 80, 129]
    w = want.copy()
    w[:, n[0] + n[1]:] = NAN
    check(s.run(q, counts, max_length=128), w, tol, "length")


def test_another_stream_and_captured():
    announce("streams and graphs")
    dtype, D = torch.float16, 64
    s = Served([700, 300], 1, D, 64, dtype, seed=9)
    q = _tensor(2 * D, 2, dtype, 56).to(DEV)
    want = s.run(q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = s.run(q)
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.zeros_like(q)
    assert torch.equal(s.run(q, stream=side, out=out), out)
    side.synchronize()
    assert torch.equal(out, want)
    # captured with the cache's writing, and replayed between eager calls
    table, lengths = s.table.to(DEV), torch.tensor(s.lengths, dtype=torch.int32, device=DEV)
    k, v = _tensor(D, 2, dtype, 57).to(DEV), _tensor(D, 2, dtype, 58).to(DEV)
    slots = torch.stack([s.slots(0, 700)[-1], s.slots(1, 300)[-1]]).to(DEV)
    prompt = [_tensor(D, 70, dtype, 59 + i).to(DEV) for i in range(3)]

    def step():
        s.cache.write(k, v, slots)
        return (s.cache.attention(q, table, lengths, max_length=700), *s.cache.read(slots), binding.window_attention(*prompt, D, window=20))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for i in range(4):
        q.copy_(_tensor(2 * D, 2, dtype, 200 + i))
        k.copy_(_tensor(D, 2, dtype, 300 + i))
        prompt[0].copy_(_tensor(D, 70, dtype, 400 + i))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        for a, b in zip(got, step()):
            assert torch.equal(a, b), i


def test_offsets_past_32_bits():
    announce("offsets past 32 bits")
    dtype, D, n = torch.float16, 64, 70
    ld = (1 << 31) // 60 + 13                                     # 64 rows span more than 4 GiB
    bufs = [torch.zeros(D * ld, dtype=dtype, device=DEV).view(D, ld) for _ in range(2)]
    q, k, v = (_tensor(D, n, dtype, 85 + i, 0.3) for i in range(3))
    views = [bufs[0][:, 11:11 + n], bufs[0][:, 100:100 + n], bufs[1][:, 11:11 + n], bufs[1][:, 100:100 + n]]
    for x, y in zip(views, (q, k, v)):
        x.copy_(y)
    binding.window_attention(*views[:3], D, out=views[3])
    check(views[3], *attend(*[x.double().numpy() for x in (q, k, v)], D, 0, dtype))
    del bufs, views
    page, heads = 1024, 16
    pages = (1 << 32) // (136 * page * heads) + 40
    cache = binding.KVCache(pages, page, heads, 128, dtype, DEV)
    k, v = _tensor(heads * 128, 40, dtype, 88), _tensor(heads * 128, 40, dtype, 89)
    cache.write(k.to(DEV), v.to(DEV), (torch.arange(40, dtype=torch.int32) + (pages - 3) * page).to(DEV))
    table = torch.tensor([[pages - 3]], dtype=torch.int32, device=DEV)
    kd, vd = (torch.from_numpy(held(x)).half().double().numpy() for x in (k, v))
    for nq in (1, 40):
        q = _tensor(heads * 128 * 2, nq, dtype, 90)
        starts = torch.tensor([0, nq], dtype=torch.int32, device=DEV)
        got = cache.attention(q.to(DEV), table, torch.tensor([40], dtype=torch.int32, device=DEV), starts, nq)
        check(got, *attend(q.double().numpy(), kd, vd, 128, 40 - nq, dtype))


@pytest.mark.parametrize("D,group,counts", [(128, 8, [8, 7, 1, 8]), (64, 5, [11, 12, 3, 10]), (96, 17, [3, 3, 1, 2]), (128, 33, [1, 1, 1, 1])])
def test_columns_in_blocks(D, group, counts):
    """More than 48 columns: blocks of whole queries, the last ones of them ragged, or not there."""
    lengths = [300, 12, 64, 101]
    s = Served(lengths, 1, D, 32, torch.bfloat16, seed=12)
    q = _tensor(group * D, sum(counts), torch.bfloat16, 64)
    for window, sinks in [(0, 0), (40, 3)]:
        announce("blocks of columns", D, group, counts, window)
        got = s.run(q, counts, window=window, sinks=sinks)
        assert "decode_kernel<%d,%d columns" % (D, 48 if group == 33 else 32) in binding.last_kernel()
        check(got, *s.want(q, counts, window=window, sinks=sinks), "window %d" % window)


def test_prompts_around_a_tile():
    """Prompts of 60 to 70 columns in all, whose last tile takes its columns from before, alone and after another."""
    for D, tokens, cut in ((64, 63, 20), (64, 64, 63), (96, 65, 64), (128, 66, 1), (64, 127, 64), (128, 129, 100)):
        announce("around a tile", D, tokens, cut)
        q, k, v = (_tensor(n * D, tokens, torch.float16, 75 + i, 0.3) for i, n in enumerate((2, 1, 1)))
        for bounds in ([0, tokens], [0, cut, tokens]):
            starts = torch.tensor(bounds, dtype=torch.int32, device=DEV)
            for window, sinks in [(0, 0), (10, 2)]:
                got = binding.window_attention(q.to(DEV), k.to(DEV), v.to(DEV), D, starts, tokens, window, sinks)
                for a, b in zip(bounds, bounds[1:]):
                    part = [x[:, a:b].double().numpy() for x in (q, k, v)]
                    check(got[:, a:b], *attend(*part, D, 0, torch.float16, window=window, sinks=sinks), "%r window %d" % (bounds, window))


@pytest.mark.parametrize("D", [64, 96, 128])
def test_short_prompts_inside_wider_rows(D):
    """Fewer than 64 columns, with NaN beside them in rows of other lengths, or rows that end where the memory does."""
    for tokens, ld, at in ((1, 1, 0), (1, 9, 4), (7, 7, 0), (9, 9, 0), (33, 40, 7), (62, 62, 0), (63, 70, 3)):
        announce("short prompt", D, tokens, ld, at)
        bufs = [torch.full((n * D, ld), NAN, dtype=torch.bfloat16, device=DEV) for n in (4, 2, 2)]
        q, k, v = (x[:, at:at + tokens] for x in bufs)
        for i, x in enumerate((q, k, v)):
            x.copy_(_tensor(x.shape[0], tokens, torch.bfloat16, 210 + i, 0.3))
        got = binding.window_attention(q, k, v, D)
        check(got, *attend(*[x.double().cpu().numpy() for x in (q, k, v)], D, 0, torch.bfloat16), "%d of %d" % (tokens, ld))
