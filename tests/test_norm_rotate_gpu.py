"""Norms of queries and keys with the rotation by position against their definition in 64 bits."""
import numpy as np
import pytest
import torch

from gpu_util import announce
from paper_2203_05016_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # relative rounding of a value, half a step
FLOOR = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}     # and of subnormals, absolute
NAN, INF = float("nan"), float("inf")


def definition(x, D, positions, frequencies, axes=None, weight=None, eps=1e-6, norm=True, interleaved=False):
    """(result, bound on how far a kernel's may be from it), both (rows, tokens) in 64 bits.

    In 32 bits the sum of D squares is off by at most D * 2^-24 of it, its root by half of that, and root, division, the factor's, the weight's and the
    rotation's products and sums by less than 16 * 2^-24 more; an angle, reduced in 64 bits to a 32-bit number of half turns, is off by 2^-25 of one,
    its sine and cosine by that times pi and two of their own steps, less than 2^-21 together.  All relative to |a| + |b| of the
    pair; then the result's rounding."""
    dtype = x.dtype
    x = x.double().cpu().numpy()
    heads, tokens, pairs = x.shape[0] // D, x.shape[1], len(frequencies)
    positions = np.atleast_2d(positions.cpu().numpy()).astype(np.float64)
    frequencies = frequencies.cpu().numpy()
    axes = np.zeros(pairs, dtype=int) if axes is None else axes.cpu().numpy()
    y = x.reshape(heads, D, tokens).copy()
    with np.errstate(all="ignore"):
        if norm:
            y = y / np.sqrt((y * y).sum(1, keepdims=True) / D + eps)
            if weight is not None:
                y = y * weight.double().cpu().numpy()[None, :, None]
        size = np.abs(y)
        first = [2 * i if interleaved else i for i in range(pairs)]
        second = [2 * i + 1 if interleaved else i + pairs for i in range(pairs)]
        known = (axes >= 0) & (axes < positions.shape[0])
        t = np.where(known[:, None], positions[np.where(known, axes, 0)] * frequencies[:, None], NAN)
        a, b = y[:, first], y[:, second]
        out, both = y.copy(), size.copy()
        out[:, first], out[:, second] = a * np.cos(t) - b * np.sin(t), a * np.sin(t) + b * np.cos(t)
        both[:, first] = both[:, second] = np.abs(a) + np.abs(b)
        tol = ((D / 2 + 16) * 2.0 ** -24 + 2.0 ** -21) * both + HALF_STEP[dtype] * np.abs(out) + FLOOR[dtype]
    return out.reshape(x.shape), tol.reshape(x.shape)


def check(got, want, what):
    """Rounding to nearest makes an infinity of what is half a step or more past the largest number: values that are by more than the
    bound past that border have to become one, those within the bound of it may."""
    dtype, (want, tol), got = got.dtype, want, got.double().cpu().numpy()
    largest = torch.finfo(dtype).max
    border = largest + 2.0 ** (np.floor(np.log2(largest))) * HALF_STEP[dtype]
    with np.errstate(invalid="ignore"):
        want = np.where(np.abs(want) > border + tol, np.copysign(INF, want), want)
        want = np.where((np.abs(np.abs(want) - border) <= tol) & np.isinf(got), np.copysign(INF, want), want)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), "%s: NaN in %d places, expected %d" % (what, np.isnan(got).sum(), nan.sum())
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), what
    ok = ~nan & ~inf
    off = np.abs(got[ok] - want[ok])
    bad = off > tol[ok]
    assert not bad.any(), "%s: %d of %d off, worst %.3e of bound" % (what, bad.sum(), bad.size, (off / tol[ok]).max())


def tensor(rows, tokens, dtype, seed, ld=None, offset=0):
    """On the GPU, with a leading dimension of its own, at an offset of its memory."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, tokens, generator=g) * torch.exp(0.5 * torch.randn(rows, 1, generator=g))).to(dtype).to(DEV)
    ld = tokens if ld is None else ld
    memory = torch.full((rows * ld + offset + 8,), 7.0, dtype=dtype, device=DEV)
    view = memory[offset:offset + rows * ld].view(rows, ld)[:, :tokens]
    view.copy_(x)
    return view


def frequencies(pairs):
    return torch.tensor([10000.0 ** (-i / max(pairs, 1)) for i in range(pairs)], dtype=torch.float64, device=DEV)


def positions(tokens, rows=1, furthest=100000, seed=0):
    g = torch.Generator().manual_seed(seed)
    p = torch.randint(-5, furthest, (rows, tokens), generator=g).to(torch.int32).to(DEV)
    return p if rows > 1 else p[0]


CASES = [  # tokens, q heads, heads, D, pairs, axes, norm, weights, interleaved, dtype
    (1, 4, 2, 64, 32, 1, True, True, False, "f16"),
    (3, 5, 1, 128, 64, 1, True, True, False, "bf16"),
    (4, 2, 2, 96, 48, 3, True, False, False, "f16"),
    (5, 16, 4, 64, 16, 1, True, True, True, "bf16"),
    (16, 3, 3, 96, 11, 2, True, True, False, "bf16"),
    (17, 8, 2, 128, 63, 1, False, False, True, "f16"),
    (63, 1, 1, 64, 32, 1, True, True, False, "f16"),
    (64, 64, 8, 128, 64, 1, True, True, False, "bf16"),
    (65, 7, 1, 96, 24, 3, True, True, False, "f16"),
    (128, 9, 3, 128, 32, 1, True, True, True, "f16"),
    (200, 2, 1, 64, 0, 1, True, True, False, "bf16"),
    (1031, 5, 5, 96, 48, 1, False, False, False, "bf16"),
    (2048, 8, 8, 128, 64, 2, True, True, False, "f16"),
    (4104, 33, 3, 64, 31, 1, True, False, True, "bf16"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c))
def test_definition(case):
    tokens, q_heads, heads, D, pairs, rows, norm, weights, interleaved, fmt = case
    announce("norm_rotate", *case)
    dtype = {"f16": torch.float16, "bf16": torch.bfloat16}[fmt]
    q, k = tensor(q_heads * D, tokens, dtype, 1), tensor(heads * D, tokens, dtype, 2)
    f, p = frequencies(pairs), positions(tokens, rows)
    axes = torch.tensor([i % rows for i in range(pairs)], dtype=torch.int32, device=DEV) if rows > 1 else None
    wq, wk = (tensor(1, D, dtype, s)[0].contiguous() if weights else None for s in (3, 4))
    kw = dict(eps=1e-5, norm=norm, interleaved=interleaved)
    got = binding.norm_rotate(q, k, D, p, f, axes=axes, q_weight=wq, k_weight=wk, **kw)
    for x, w, y in zip((q, k), (wq, wk), got):
        assert y.shape == x.shape and y.dtype == dtype
        check(y, definition(x, D, p, f, axes, w, **kw), case)


@pytest.mark.parametrize("tokens", [2, 15, 64, 67, 256])
@pytest.mark.parametrize("ld,offset", [(0, 0), (3, 0), (8, 1), (8, 8), (40, 4)])
def test_strides_and_what_lies_around(tokens, ld, offset):
    announce("norm_rotate strides", tokens, ld, offset)
    D, dtype = 64, torch.float16
    q, k = tensor(4 * D, tokens, dtype, 1, tokens + ld, offset), tensor(2 * D, tokens, dtype, 2, tokens + 2 * ld, offset)
    f, p, w = frequencies(32), positions(tokens), tensor(1, D, dtype, 3)[0].contiguous()
    want = [definition(x, D, p, f, weight=w) for x in (q, k)]
    plain = binding.norm_rotate(q.contiguous(), k.contiguous(), D, p, f, q_weight=w, k_weight=w)
    memory = [torch.full((rows * (tokens + ld) + offset + 8,), 3.0, dtype=dtype, device=DEV) for rows in (4 * D, 2 * D)]
    outs = [m[offset:-8].view(-1, tokens + ld)[:, :tokens] for m in memory]
    got = binding.norm_rotate(q, k, D, p, f, q_weight=w, k_weight=w, q_out=outs[0], k_out=outs[1])
    for y, out, x, same, m in zip(got, outs, want, plain, memory):
        assert y is out and torch.equal(y, same)
        check(y, x, (tokens, ld, offset))
        body = m[offset:-8].view(-1, tokens + ld)
        assert (body[:, tokens:] == 3).all() and (m[:offset] == 3).all() and (m[-8:] == 3).all()
    for x in (q, k):                                            # in place
        around = x._base.clone()
        around.as_strided(x.shape, x.stride(), x.storage_offset()).copy_(plain[0] if x is q else plain[1])
        if x is k:
            binding.norm_rotate(q, k, D, p, f, q_weight=w, k_weight=w, q_out=q, k_out=k)
            assert torch.equal(q, plain[0]) and torch.equal(k, plain[1]) and torch.equal(k._base, around)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tokens", [3, 70, 72])
def test_values_at_their_limits(tokens, dtype):
    """Infinities and NaN stay in their head and token; squares beyond 32 bits; nothing but zeros."""
    announce("norm_rotate limits", tokens, dtype)
    D = 128
    q = tensor(4 * D, tokens, dtype, 5)
    q[5, 0], q[D + 7, 1], q[2 * D:3 * D, 2] = INF, NAN, 0
    big = 60000.0 if dtype == torch.float16 else 2.0 ** 125
    q[3 * D:, 0] *= 2.0 ** -20 if dtype == torch.float16 else 2.0 ** -100
    q[3 * D:, 1] = q[3 * D:, 1].clamp(-1, 1) * big
    f, p = frequencies(64), positions(tokens)
    for eps in (0.0, 1e-6, 2.0 ** -150):
        got, none = binding.norm_rotate(q, None, D, p, f, eps=eps)
        assert none is None
        check(got, definition(q, D, p, f, eps=eps), (tokens, dtype, eps))
    turned, _ = binding.norm_rotate(q, None, D, p, f, norm=False)
    check(turned, definition(q, D, p, f, norm=False), (tokens, dtype))


def test_far_positions_and_rows_that_are_not_there():
    announce("norm_rotate far positions")
    D, tokens, dtype = 64, 96, torch.float16
    q = tensor(2 * D, tokens, dtype, 6)
    f = frequencies(32)
    p = torch.tensor([2 ** 31 - 1 - i if i % 2 else i - 2 ** 31 for i in range(tokens)], dtype=torch.int32, device=DEV)
    got, _ = binding.norm_rotate(q, None, D, p, f)
    check(got, definition(q, D, p, f), "far")
    axes = torch.tensor([(-1, 0, 1, 2, 2 ** 31 - 1)[i % 5] for i in range(32)], dtype=torch.int32, device=DEV)
    two = positions(tokens, 2)
    got, _ = binding.norm_rotate(q, None, D, two, f, axes=axes)
    check(got, definition(q, D, two, f, axes), "axes")
    assert torch.isnan(got).any() and not torch.isnan(got).all()


def test_rotation_keeps_products_of_equal_distance():
    """What the rotation is for: q.k depends on the difference of positions alone."""
    announce("norm_rotate distances")
    D, dtype, f = 128, torch.float16, frequencies(64)
    q, k = tensor(D, 1, dtype, 8).expand(D, 64).contiguous(), tensor(D, 1, dtype, 9).expand(D, 64).contiguous()
    p = (torch.arange(64, device=DEV) * 977).int()
    turned = binding.norm_rotate(q, k, D, p, f)
    moved = binding.norm_rotate(q, k, D, p + 12345, f)
    product = lambda x: (x[0].double().t().contiguous() @ x[1].double()).cpu()
    a, b = product(turned), product(moved)
    # each of 2 * 128 factors of both sums is off by half a step (2^-11) and 2^-17 of arithmetic, relative to columns of norm sqrt(128)
    assert (a - b).abs().max() <= 4 * 128 * (2.0 ** -11 + 2.0 ** -17)
    assert (a[0] - a[0, 0]).abs().max() > 1


def test_rows_that_are_far_apart():
    """Offsets past 32 bits: rows of 2^23 tokens and more, of which a few thousand are taken, where runs of 16 bytes are not, and 2^25 of a head's bytes apart."""
    announce("norm_rotate far rows")
    D, dtype, f = 64, torch.float16, frequencies(32)
    for ld, tokens in (((1 << 23) + 40, 19000), ((1 << 23) - 8, 9001)):
        memory = torch.zeros(3 * D * ld, dtype=dtype, device=DEV)
        rows = memory.view(3 * D, ld)[:, ld - tokens:]              # the last columns
        x = tensor(3 * D, tokens, dtype, 3)
        rows.copy_(x)
        p = positions(tokens)
        q, k = rows[:2 * D], rows[2 * D:]
        want = binding.norm_rotate(x[:2 * D], x[2 * D:], D, p, f)
        binding.norm_rotate(q, k, D, p, f, q_out=q, k_out=k)
        for got, y in ((q, want[0]), (k, want[1])):
            # each is within definition's bound; a column's squares add up to D, so |a| + |b| is at most (2 D)^0.5
            off = 2 * (2.0 ** -11 * 1.001 * y.double().abs() + ((D / 2 + 16) * 2.0 ** -24 + 2.0 ** -21) * (2 * D) ** 0.5 + 2.0 ** -25)
            assert ((got.double() - y.double()).abs() <= off).all()
        check(q[:D, -50:], definition(x[:D, -50:], D, p[-50:], f), "far rows")
        assert (memory.view(3 * D, ld)[:, :ld - tokens] == 0).all()
        del memory, rows, q, k


def test_nothing_to_do():
    announce("norm_rotate nothing")
    f = frequencies(32)
    none = torch.zeros(128, 0, dtype=torch.float16, device=DEV)
    q, k = binding.norm_rotate(none, none, 64, torch.zeros(0, dtype=torch.int32, device=DEV), f)
    assert q.shape == k.shape == (128, 0)


def test_graph_and_streams():
    """Captured and replayed with other inputs between, and on another stream."""
    announce("norm_rotate graph")
    D, tokens, dtype = 96, 48, torch.bfloat16
    q, k = tensor(4 * D, tokens, dtype, 1), tensor(2 * D, tokens, dtype, 2)
    f, p = frequencies(48), positions(tokens)
    call = lambda **kw: binding.norm_rotate(q, k, D, p, f, **kw)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = call()
    for seed in range(3):
        q.copy_(tensor(4 * D, tokens, dtype, 10 + seed))
        p.copy_(positions(tokens, seed=seed))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, call()))
    side = torch.cuda.Stream()
    want = call()
    torch.cuda.synchronize()
    got = call(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
