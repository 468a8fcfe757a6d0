"""Attention where a call's bounds and its tensors' values are at their limits, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from attention_reference import HALF_STEP, attend, check
from gpu_util import announce
from paper_2203_05016_amd import binding
from test_attention_gpu import DEV, INF, NAN, Served, _tensor

pytestmark = pytest.mark.gpu


def _starts(counts):
    return torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("D,heads,group,counts", [
    (128, 8, 8, [1] * 32), (128, 8, 8, [40] + [0] * 63), (128, 16, 8, [3] * 16), (128, 16, 5, [3] * 20), (128, 32, 8, [7] * 8),
    (96, 16, 8, [2] * 31), (64, 16, 8, [2] * 31), (128, 8, 8, [63] + [0] * 40)])
def test_short_prompts_of_many_sequences(D, heads, group, counts):
    """Fewer than 64 columns in all, and more workgroups than the GPU has CUs: every query head and query is computed."""
    announce("short prompts", D, heads, group, len(counts), max(counts))
    tokens = sum(counts)
    q, k, v = (_tensor(n * D, tokens, torch.bfloat16, 60 + i, 0.5 if i < 2 else 0) for i, n in enumerate((heads * group, heads, heads)))
    out = torch.full((heads * group * D, tokens), NAN, dtype=torch.bfloat16, device=DEV)
    binding.window_attention(q.to(DEV), k.to(DEV), v.to(DEV), D, _starts(counts), max(counts), out=out)
    at = 0
    for n in counts:
        if n:
            part = [x[:, at:at + n].double().numpy() for x in (q, k, v)]
            check(out[:, at:at + n], *attend(*part, D, 0, torch.bfloat16), "columns %d to %d" % (at, at + n - 1))
        at += n


@pytest.mark.parametrize("counts,max_length,parts", [(None, 64, False), (None, 1, False), (None, 2100, True), ([5, 3], 100, False), ([5, 3], 2100, True),
                                                     ([80, 41], 100, False), ([80, 41], 1000, True)])
@pytest.mark.parametrize("D,group", [(64, 4), (128, 8)])
def test_lengths_past_max_length(D, group, counts, max_length, parts):
    """max_length decides how the work is cut, never what is computed: sequences that have grown past it see all their keys."""
    announce("past max_length", D, group, counts, max_length)
    s = Served([3500, 2777], 1, D, 64, torch.float16, seed=14)
    q = _tensor(group * D, sum(counts) if counts else 2, torch.float16, 66)
    seqs = binding._Sequences(group, 2, max(counts or [1]), s.table.shape[1], 0, 0, q.shape[1], max_length, s.table.shape[1], None, None, 1 if counts else None)
    assert (binding.lib().shflbw_kv_attention_workspace(s.cache._c, seqs) > 0) == parts
    for window, sinks in [(0, 0), (2200, 70)]:
        got = s.run(q, counts, window=window, sinks=sinks, max_length=max_length)
        check(got, *s.want(q, counts or [1, 1], window=window, sinks=sinks), "window %d" % window)


@pytest.mark.parametrize("counts", [[5, 3], [80, 41]])
def test_a_generous_bound_of_queries(counts):
    announce("generous max_queries", counts)
    D, group = 64, 4
    s = Served([250, 177], 1, D, 64, torch.bfloat16, seed=16)
    q = _tensor(group * D, sum(counts), torch.bfloat16, 68).to(DEV)
    table, lengths = s.table.to(DEV), torch.tensor(s.lengths, dtype=torch.int32, device=DEV)
    want = s.cache.attention(q, table, lengths, _starts(counts), max_queries=sum(counts))
    check(want, *s.want(q.cpu(), counts))
    for most in (1000, 2 ** 31 - 1):
        assert torch.equal(want, s.cache.attention(q, table, lengths, _starts(counts), max_queries=most))


@pytest.mark.parametrize("counts", [None, [5, 3], [80, 41]])
@pytest.mark.parametrize("dtype,byte", [(torch.float16, 200), (torch.float16, 254), (torch.bfloat16, 254)])
@pytest.mark.parametrize("D", [64, 128])
def test_slots_that_were_never_written(D, dtype, byte, counts):
    """They hold what was there: here codes and scales whose values 16 bits cannot hold, which no query sees."""
    announce("never written", D, dtype, byte, counts)
    s = Served([250, 177], 2, D, 32, dtype, seed=15)
    s.cache._dev.fill_(byte)
    for b, n in enumerate(s.lengths):
        s.put(b, _tensor(2 * D, n, dtype, 400 + b), _tensor(2 * D, n, dtype, 500 + b, 0))
    q = _tensor(4 * D, sum(counts) if counts else 2, dtype, 67)
    for window, sinks in [(0, 0), (70, 5)]:
        got = s.run(q, counts, window=window, sinks=sinks)
        check(got, *s.want(q, counts or [1, 1], window=window, sinks=sinks), "window %d" % window)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D,group", [(64, 2), (96, 2), (128, 8)])
@pytest.mark.parametrize("steep", [1, 10])
def test_infinite_values_of_next_to_no_weight(dtype, D, group, steep):
    """An infinity among the values a query sees is its result's, however small its weight and wherever its key lies: weights that
    16 or 32 bits hold as zero, before the maximum (that the accumulators are scaled down for) and after it."""
    n, step = 420, 14.0 if dtype == torch.float16 else 12.0
    q, k, v = torch.full((group * D, n), steep * step / D ** 0.5, dtype=dtype), torch.zeros(D, n, dtype=dtype), _tensor(D, n, dtype, 33, 0)
    top, deep = 200, 300                                  # scores: 0, at `top` that much more, at `deep` that much less
    k[:, top], k[:, deep] = 8 / D ** 0.5, -8 / D ** 0.5
    v[3, 10], v[17, deep], v[40, 10], v[40, deep], v[50, 350], v[60, 5] = INF, -INF, INF, -INF, NAN, -INF
    clean = torch.where(torch.isfinite(v), v, 0)
    for window, sinks in [(0, 0), (260, 0), (130, 8)]:
        announce("infinite values", dtype, D, group, steep, window, sinks)
        got = binding.window_attention(q.to(DEV), k.to(DEV), v.to(DEV), D, window=window, sinks=sinks)
        want, tol = attend(*[x.double().numpy() for x in (q, k, clean)], D, 0, dtype, window=window, sinks=sinks)
        p, j = np.arange(n)[:, None], np.arange(n)[None]
        seen = (j <= p) & ((j > p - window) | (j < sinks) if window else True)
        for f in (3, 17, 40, 50, 60):
            special = np.where(torch.isfinite(v[f]).numpy(), 0, v[f].double().numpy())
            with np.errstate(invalid="ignore"):
                total = np.array([special[s].sum() for s in seen])
            for h in range(group):
                row = want[h * D + f]
                row[total != 0] = total[total != 0]
        check(got, want, tol, "window %d sinks %d" % (window, sinks))


@pytest.mark.parametrize("D", [64, 128])
def test_many_small_weights(D):
    """One key of much weight and tens of thousands of 2^-26 of it: the sum of the weights and that of the weighted values leave none out.

    Bound: a weight's rounding to binary16 is off by 2^-11 of it, or, of weights 2^6 times as large, by 2^-25 where they are subnormal: 2^-31
    beside the largest; sums, exponentials and scores as in attention_reference."""
    announce("small weights", D)
    n, dtype = 40000, torch.float16
    c = 26 * np.log(2.0)                                  # the first key's score beside the others' zeros
    q = torch.full((D, n), c / D ** 0.5, dtype=dtype)
    k, v = torch.zeros(D, n, dtype=dtype), torch.ones(D, n, dtype=dtype)
    k[:, 0], v[:, 0] = 1, 0
    got = binding.window_attention(q.to(DEV), k.to(DEV), v.to(DEV), D)
    for p in (0, 1, 1000, 20000, 39999):
        score = float(q[0, p].double()) * D ** 0.5
        rest = p * np.exp(-score)
        want = rest / (1 + rest)
        tol = p * 2.0 ** -31 + want * (2 * HALF_STEP[dtype] + 2 * ((D + 4) * 2.0 ** -24 * score + 2.0 ** -22) + 2 * n * 2.0 ** -24) + 2.0 ** -25
        off = (got[:, p].double() - want).abs().max().item()
        assert off <= tol, (p, off, tol, want)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_up_to_sixteen_million(dtype, D):
    """Scores whose steps in 32 bits are as large as 1, of both signs: which keys they pick is left open, but values that are the same for all
    keys are what any weights give.  Bound: the weights' rounding (half a step above and below), the sum's of n of them, the result's."""
    n, group = 300, 2
    size = (1.5e7 / D ** 0.5) ** 0.5
    g = torch.Generator().manual_seed(41)
    rand = lambda rows: (size * (1 - torch.rand(rows, n, generator=g) / 64)).to(dtype)
    q, k = rand(group * D), rand(D)
    q[:, ::2] *= -1
    v = (torch.rand(D, 1, generator=g) + 0.5).to(dtype).expand(D, n).contiguous()
    assert 1e7 < float(q.double()[:D].abs().mul(k.double()).sum(0).max()) / D ** 0.5 < 1.6e7
    announce("large scores", dtype, D)
    tol = 3 * HALF_STEP[dtype] + 2 * n * 2.0 ** -24
    got = binding.window_attention(q.to(DEV), k.to(DEV), v.to(DEV), D).double().cpu()
    want = v.double().repeat(group, 1)
    assert bool(((got - want).abs() <= tol * want).all()), ((got - want).abs() / want).max()
    s = Served([n], 1, D, 32, dtype, seed=17)
    s.put(0, k, v)
    want = torch.from_numpy(s.v[0])[:, -1:].repeat(group, 1)
    for nq in (1, 3, 90):
        got = s.run(q[:, -nq:], [nq]).double().cpu()
        assert bool(((got - want).abs() <= tol * want).all()), (nq, ((got - want).abs() / want).max())
