"""The attention operators' definition in 64 bits on the CPU, and how far a result may be from it."""
import numpy as np
import torch

HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # relative rounding of a value, half a step
FLOOR = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}             # and of subnormals, absolute
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def held(x):
    """What the cache holds of the (rows, tokens) tensor x, in 64 bits: 32 rows of a column are a block."""
    a = x.double().numpy()
    out = np.empty_like(a)
    for i in range(0, a.shape[0], 32):
        for t in range(a.shape[1]):
            block = a[i:i + 32, t]
            if not np.isfinite(block).all():
                out[i:i + 32, t] = np.nan
                continue
            largest = np.abs(block).max()
            e = max(int(np.frexp(largest)[1]) - 3, -126) if largest else -126
            r = np.abs(block) / 2.0 ** e
            d = np.abs(r[:, None] - GRID[None])
            best = d.min(1)
            pick = np.empty(32, dtype=int)
            for n in range(32):
                near = np.nonzero(d[n] == best[n])[0]
                pick[n] = near[0] if len(near) == 1 or near[0] % 2 == 0 else near[1]
            out[i:i + 32, t] = np.copysign(GRID[pick], block) * 2.0 ** e
    return out


def attend(q, k, v, head_dim, first, dtype, window=0, sinks=0):
    """q (q_heads * head_dim, n) at positions first and up, k and v (heads * head_dim, keys), 64-bit arrays.  Returns the result and,
    element by element, how far a kernel's result of `dtype` may be from it.

    With w the weights before the division and W = sum(w |v|) / sum(w), a kernel's result is off by at most
      * scores: products of 16-bit values are exact in 32 bits, their sum of head_dim terms is off by head_dim * 2^-24 of the sum of
        magnitudes A, scaling and the subtraction of the maximum by 4 * 2^-24 of it, the exponential by 2^-22: a weight is off by
        (head_dim + 4) * 2^-24 * A + 2^-22 relatively, the result by twice that times W (numerator and denominator)
      * the weights' rounding to dtype: half a step times W, and 2^-25 per key where they are subnormal binary16 (the
        largest weight is 1, so the sum is at least 1)
      * sums over n keys: 2 n 2^-24 W, accumulators included; joins of parts 2^-20 W
      * the result's rounding."""
    D, heads, group = head_dim, k.shape[0] // head_dim, q.shape[0] // k.shape[0]
    n, keys = q.shape[1], k.shape[1]
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    j = np.arange(keys)
    for h in range(heads * group):
        kh, vh = (x[h // group * D:(h // group + 1) * D] for x in (k, v))
        for i in range(n):
            p = first + i
            seen = (j <= p) & ((j > p - window) | (j < sinks) if window else True)
            if p < 0 or not seen.any():
                continue
            qi, ks, vs = q[h * D:(h + 1) * D, i], kh[:, seen], vh[:, seen]
            with np.errstate(invalid="ignore", over="ignore"):
                s = qi @ ks / np.sqrt(D)
                A = (np.abs(qi) @ np.abs(ks) / np.sqrt(D)).max()
                w = np.exp(s - s.max())
                o = vs @ w / w.sum()
                W = np.abs(vs) @ w / w.sum()
                off = 2 * ((D + 4) * 2.0 ** -24 * A + 2.0 ** -22) + HALF_STEP[dtype] + 2 * seen.sum() * 2.0 ** -24 + 2.0 ** -20
                t = off * W + HALF_STEP[dtype] * np.abs(o) + FLOOR[dtype] * (1 + seen.sum() * np.abs(vs).max())
            out[h * D:(h + 1) * D, i], tol[h * D:(h + 1) * D, i] = o, t
    return out, tol


def check(got, want, tol, what=""):
    got = got.double().cpu().numpy()
    assert got.shape == want.shape
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), "%s: NaN in %d places, expected %d" % (what, np.isnan(got).sum(), nan.sum())
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), what
    ok = ~nan & ~inf
    off = np.abs(got[ok] - want[ok])
    bad = off > tol[ok]
    assert not bad.any(), "%s: %d of %d off, worst %.3e of bound" % (what, bad.sum(), bad.size, (off / np.maximum(tol[ok], 1e-300)).max())
