"""How far the result of an 8-bit product may be from 64 bits as a whole: far less than what each of its values may be off (q8_reference.py).

What is off in a sum is taken as so many independent errors, and their squares are added:
  * fp32 sums: k additions, each off by at most half a step, 2^-24, of a partial sum.  The mean square of the partial sum of j of k terms of unlike signs is j / k
    of the last one's, so k / 2 of those, a third of the square for an error that lies anywhere within: (k / 6) 2^-48 of the sum's square.  Taken as
    k 2^-48, as no order of additions and no distribution of the signs is known: sqrt(k) 2^-24 of the sums' 2-norm.
  * dtype bf16 and 8-bit results of it: besides, eight neighbouring products are added at a time, each of the seven others cut off less than 2^-13 below the
    exponent of the largest, somewhere within: a third of its square, 7 / 3 (2^-13 max)^2 a group.
Then the last rounding.  With fp32 it is 2^-24 of the result, and added.  With fewer bits it hides all that (its own part of the 2-norm is 1.7 10^-3), and in 2-norm a few
large values that come out a step away are more than all others; so the values that are not the correctly rounded ones are counted.  One that is d off comes out another with
probability |d| / step, of which the mean is at most the root of the mean square over the step; so many are expected in all, with at most that variance, and four standard
deviations more are allowed.  Values whose steps are below four times what they may be off, by chance next to zero, say nothing.
"""
import numpy as np

import q8_reference as ref

U = 2.0 ** -24


def cut_off(a, w):
    """Mean square of what is cut off of each sum."""
    m, n, k = a.shape[0], w.shape[0], a.shape[1]
    a8, w8 = np.abs(a).reshape(m, k // 8, 8).astype(np.float32), np.abs(w).reshape(n, k // 8, 8).astype(np.float32)
    out = np.zeros((m, n))
    for g in range(k // 8):
        top = np.zeros((m, n), np.float32)
        for i in range(8):
            np.maximum(top, a8[:, g, i, None] * w8[None, :, g, i], out=top)
        out += top.astype(np.float64) ** 2
    return out * (7 / 3) * 2.0 ** -26


def sums(a, w, dtype):
    """The sums, and the root of the mean square of what each is off by."""
    z = a @ w.T
    sq = z * z                  # (a sum may be small by chance, its terms are as large as its row's and column's others)
    d = a.shape[1] * U * U * sq.mean(1, keepdims=True) * sq.mean(0, keepdims=True) / sq.mean()
    return z, np.sqrt(d + cut_off(a, w) if dtype == "bf16" else d)


def linear(a, w, dtype, up=None, bias=None, relu=False, residual=None):
    """The result in 64 bits and what each value is off by before the last rounding."""
    z, d = sums(a, w, dtype)
    if bias is not None:
        z = z + bias
        d = np.hypot(d, U * z)
    if relu:
        z = np.maximum(z, 0)
    if up is not None:
        u, d_u = sums(a, up, dtype)
        s = ref.silu(z)
        with np.errstate(over="ignore"):
            slope = 1 / (1 + np.exp(-z)) * (1 + z / (1 + np.exp(z)))
        z, d = s * u, np.sqrt((slope * d * u) ** 2 + (s * d_u) ** 2 + ((np.abs(z) + 8) * 2 * U * s * u) ** 2)
    if residual is not None:
        z = z + residual
        d = np.hypot(d, U * z)
    return z, d


def round_bf16(x):
    """Nearest, ties to even, of float64 (normal numbers)."""
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -126))) - 7)
    return np.rint(x / step) * step, step


def count(got, near, step, d, what):
    """Values that are not the correctly rounded ones."""
    sure = step >= 4 * d
    assert sure.mean() > 0.5, "what may be off hides the rounding"
    off, expected = (got != near)[sure].sum(), (d / step)[sure].sum()
    assert off <= expected + 4 * np.sqrt(expected), f"{what}: {off} of {sure.sum()} values are not the nearest, {expected:.0f} are expected at most"


def check_rows(got, want, d, dtype, what=""):
    got = np.asarray(got, np.float64)
    if dtype == "bf16":
        return count(got, *round_bf16(want), d, what)
    off, allowed = np.linalg.norm(got - want), np.linalg.norm(d) + U * np.linalg.norm(want)
    assert off <= allowed, f"{what}: off by {off / np.linalg.norm(want):.3e} in 2-norm, {allowed / np.linalg.norm(want):.3e} is allowed"


def check_held(codes, scales, want, d, what=""):
    near, near_scales = ref.hold(want)
    count(ref.values(codes, scales), ref.values(near, near_scales), 2 * ref.half_steps(want, near_scales), d, what)
