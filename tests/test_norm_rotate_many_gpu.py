"""Norms with rotation of many tokens, in the forms that only large calls take: 32 tokens to a wavefront with results past the L2s (rows of whole 64 bytes,
16 MB of them), 64 to a wavefront (other rows, 300000 columns of heads and more), several rounds of heads to a workgroup, heads of 96; and what
these do with values that 32 bits do not hold.  Heads repeat a few, so that the definition is worked out for those alone: a head's
result depends on nothing but its own values, weights, tokens' positions."""
import numpy as np
import pytest
import torch

from gpu_util import announce
from paper_2203_05016_amd import binding
from test_norm_rotate_gpu import DEV, INF, NAN, check, definition, frequencies, positions, tensor

pytestmark = pytest.mark.gpu
DISTINCT = 7                        # heads; nothing in the kernels goes by 7
F16, BF16 = torch.float16, torch.bfloat16


def repeated(base, D, heads, first, ld, offset):
    """`heads` heads, head h being the (first + h)-th of base's, in memory of its own pitch, at an offset."""
    tokens = base.shape[1]
    pick = [(first + h) % DISTINCT for h in range(heads)]
    memory = torch.full((heads * D * ld + offset + 8,), 7.0, dtype=base.dtype, device=DEV)
    view = memory[offset:offset + heads * D * ld].view(heads * D, ld)[:, :tokens]
    view.copy_(base.view(DISTINCT, D, tokens)[pick].reshape(heads * D, tokens))
    return view, pick, memory


def compare(got, pick, D, want, what):
    """The first of every distinct head against its definition, all others against the first, bit for bit (NaN as NaN)."""
    heads, first = got.view(len(pick), D, got.shape[1]) if got.is_contiguous() else got.unflatten(0, (len(pick), D)), {}
    value, tol = want
    for h, n in enumerate(pick):
        if n not in first:
            first[n] = h
            rows = slice(n * D, n * D + D)
            check(heads[h], (value[rows], tol[rows]), what + (h,))
        else:
            assert torch.equal(heads[h].view(torch.int16) if heads[h].is_contiguous() else heads[h].contiguous().view(torch.int16),
                               heads[first[n]].contiguous().view(torch.int16)), what + (h,)


CASES = [  # tokens, q heads, heads, D, pairs, pitch past the tokens, offset, in place, interleaved, dtype
    (8192, 64, 8, 128, 64, 0, 0, False, False, "bf16"),     # whole rows, past the L2s, two rounds of heads
    (8192, 66, 7, 64, 20, 32, 0, True, True, "f16"),        # the same in place, behind a pitch
    (2080, 40, 3, 96, 48, 0, 0, False, False, "f16"),       # past the L2s
    (640, 40, 2, 96, 40, 0, 0, False, True, "bf16"),        # whole rows, through the L2s
    (643, 30, 5, 96, 48, 0, 0, True, False, "f16"),         # others, 32 tokens to a wavefront
    (1021, 16, 3, 128, 64, 3, 1, True, False, "bf16"),
    (4171, 64, 8, 128, 64, 0, 0, False, False, "bf16"),     # others, 64 tokens to a wavefront
    (4171, 64, 9, 128, 31, 5, 3, True, True, "f16"),
    (5003, 57, 4, 96, 48, 1, 0, True, False, "bf16"),
    (3777, 73, 8, 64, 32, 2, 7, False, False, "f16"),
    (16383, 64, 8, 64, 32, 0, 0, True, False, "bf16"),      # the same, two rounds of heads
    (8192, 36, 1, 96, 48, 0, 1, False, False, "f16"),       # rows of whole 64 bytes that begin at no line
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c))
def test_definition(case):
    tokens, q_heads, heads, D, pairs, pitch, offset, in_place, interleaved, fmt = case
    announce("norm_rotate, many", *case)
    dtype = {"f16": F16, "bf16": BF16}[fmt]
    base = tensor(DISTINCT * D, tokens, dtype, 1)
    wq, wk = (tensor(1, D, dtype, s)[0].contiguous() for s in (3, 4))
    f, p = frequencies(pairs), positions(tokens)
    want = [definition(base, D, p, f, None, w, 1e-5, True, interleaved) for w in (wq, wk)]
    ins = [repeated(base, D, n, first, tokens + pitch, offset) for n, first in ((q_heads, 0), (heads, 3))]
    outs = [x[0] for x in ins]
    memories = [x[2] for x in ins]
    if not in_place:
        memories = [torch.full_like(x[2], 7.0) for x in ins]
        outs = [m[offset:offset + x[0].shape[0] * (tokens + pitch)].view(-1, tokens + pitch)[:, :tokens] for m, x in zip(memories, ins)]
    got = binding.norm_rotate(ins[0][0], ins[1][0], D, p, f, q_weight=wq, k_weight=wk, eps=1e-5, interleaved=interleaved, q_out=outs[0], k_out=outs[1])
    for y, out, (_, pick, _), x, m in zip(got, outs, ins, want, memories):
        assert y is out
        compare(y, pick, D, x, case)
        body = m[offset:offset + y.shape[0] * (tokens + pitch)].view(-1, tokens + pitch)
        assert (body[:, tokens:] == 7).all() and (m[:offset] == 7).all() and (m[-8:] == 7).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("tokens,pitch,D", [(1024, 0, 128), (1027, 0, 128), (1027, 5, 96), (8192, 0, 64), (4171, 0, 128), (5003, 1, 64)])
@pytest.mark.parametrize("in_place", [False, True])
def test_values_at_their_limits(tokens, pitch, D, dtype, in_place):
    """Infinities and NaN stay in their head and token; squares beyond 32 bits on either side; nothing but zeros: in the first tokens, in those that the last
    runs share with the runs before them, and between."""
    announce("norm_rotate, many, limits", tokens, pitch, D, dtype, in_place)
    base = tensor(DISTINCT * D, tokens, dtype, 5)
    half = dtype == F16
    for at in (0, 37, 511, tokens - 1, tokens - 4, tokens - 9, tokens - 65):
        base[5, at], base[D + 7, at], base[2 * D:3 * D, at] = INF, NAN, 0
        base[3 * D:4 * D, at] *= 2.0 ** -20 if half else 2.0 ** -100
        base[4 * D:5 * D, at] = base[4 * D:5 * D, at].clamp(-1, 1) * (60000.0 if half else 2.0 ** 125)
        base[5 * D:6 * D, at] *= 2.0 ** -12 if half else 2.0 ** -33                     # squares whose sum is near 2^-60 (binary16: small)
    heads = (64, 9)
    f, p, w = frequencies(D // 2), positions(tokens), tensor(1, D, dtype, 3)[0].contiguous()
    for eps in (0.0, 1e-6, 2.0 ** -150):
        want = definition(base, D, p, f, weight=w, eps=eps)
        ins = [repeated(base, D, n, first, tokens + pitch, 0) for n, first in zip(heads, (0, 3))]
        outs = [x[0] if in_place else torch.empty_like(x[0]) for x in ins]
        got = binding.norm_rotate(ins[0][0], ins[1][0], D, p, f, q_weight=w, k_weight=w, eps=eps, q_out=outs[0], k_out=outs[1])
        for y, (_, pick, _) in zip(got, ins):
            compare(y, pick, D, want, (tokens, D, dtype, in_place, eps))


def test_nothing_depends_on_the_form():
    """Tokens in the middle of a large call and alone: by other kernels, within both bounds of the definition."""
    announce("norm_rotate, forms")
    D, tokens, dtype = 128, 4171, BF16
    base, f, p = tensor(DISTINCT * D, tokens, dtype, 1), frequencies(64), positions(tokens)
    q, pick, _ = repeated(base, D, 72, 0, tokens, 0)
    got, _ = binding.norm_rotate(q, None, D, p, f)
    few = slice(1000, 1003)
    alone, _ = binding.norm_rotate(base[:, few], None, D, p[few], f)
    want = definition(base[:, few], D, p[few], f)
    check(alone, want, "alone")
    check(got[:DISTINCT * D, few], want, "among others")
    assert np.isfinite(want[0]).all()
