"""The user cache in 64 bits (include/aif_cache.h): what a row stands for once it is held in 4 bits, and attention over it."""
import numpy as np

BLOCK = 32
MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)


def hold(x):
    """x [..., d] -> the values its codes and scales stand for, float64."""
    x = np.asarray(x, np.float64)
    out = np.empty_like(x)
    for lo in range(0, x.shape[-1], BLOCK):
        b = x[..., lo:lo + BLOCK]
        with np.errstate(invalid="ignore"):
            top = np.abs(b).max(-1, keepdims=True)          # NaN where there is one
        finite = np.isfinite(top)
        f, e = np.frexp(np.where(finite, top, 0.0))         # top = f 2^e, f in [1/2, 1)
        e = np.clip(np.where(f <= 0.75, e - 3, e - 2), -125, 125)
        e = np.where(top == 0, -125, e)
        a = np.abs(np.where(finite, b, 0.0)) / np.exp2(e.astype(np.float64))
        off = np.abs(a[..., None] - MAGNITUDES)             # nearest; of two equally near the one at an even place
        near = off.min(-1, keepdims=True)
        place = np.where(off == near, np.where(np.arange(8) % 2 == 0, 0, 1), 2).argmin(-1)
        v = np.copysign(MAGNITUDES[place] * np.exp2(e.astype(np.float64)), b)
        out[..., lo:lo + BLOCK] = np.where(finite, v, np.nan)
    return out


def sees(n_keys, positions, sinks, window, dropped=()):
    """[n_q, n_keys] truth values; dropped: (first, end) runs of rows that were dropped."""
    j = np.arange(n_keys)[None, :]
    p = np.asarray(positions, np.int64)[:, None]
    see = j <= p
    if window:
        see = see & ((j > p - window) | (j < sinks))
    for lo, hi in dropped:
        see = see & ~((j >= lo) & (j < hi))
    return see


def attend(q, keys, vals, scale, see):
    """q [n_q, H, d], keys and vals [n, H_kv, d] (held), see [n_q, n].  Returns out [n_q, H, d], lse [n_q, H] and, for the
    tolerances, the weighted sum of the values' magnitudes [n_q, H, d] and per row the largest sum of |q||k| scale and of |score| [n_q, H]."""
    q = np.asarray(q, np.float64)
    n_q, heads, d = q.shape
    group = heads // keys.shape[1]
    out, mag = np.zeros((n_q, heads, d)), np.zeros((n_q, heads, d))
    lse, big, top = np.full((n_q, heads), -np.inf), np.zeros((n_q, heads)), np.zeros((n_q, heads))
    any_key = see.any(1)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        for h in range(heads):
            k, v = keys[:, h // group], vals[:, h // group]
            s = q[:, h] @ k.T * scale
            for i in np.flatnonzero(any_key):
                at = np.flatnonzero(see[i])
                si = s[i, at]
                m = si.max()
                if m == -np.inf:
                    continue
                w = np.exp(si - m)
                lse[i, h] = m + np.log(w.sum())
                out[i, h] = (w[:, None] * v[at]).sum(0) / w.sum()
                mag[i, h] = (w[:, None] * np.abs(v[at])).sum(0) / w.sum()
                big[i, h] = (np.abs(q[i, h]) @ np.abs(k[at]).T).max() * scale
                top[i, h] = np.abs(si).max()
    return out, lse, mag, big, top


def tolerances(dtype, d, n, out, lse, mag, big, top):
    """(for out, for lse).  u = 2^-24 is half a step of fp32.  A score is a sum of d products, one more rounding scales it:
    off by at most (d + 2) u big, taken from the maximum and put through exp2 (argument u (|s| + |m|) log2 e, the instruction
    2 u): a weight is relatively off by 2 ((d + 2) big + 2 top + 2) u at most.  The sums over n keys add n u, and as much again the
    running maximum's corrections (each a product, at most one a key).  In fp32 a weight and a query are three bf16 pieces, exact to
    2^-24 u.  In bf16 the weights are rounded to bf16, 2^-8 relative, and so is the output."""
    u = 2.0 ** -24
    weight = 2 * ((d + 2) * big + 2 * top + 2) * u
    rel = (weight + (2 * n + 4) * u)[..., None]
    tol = rel * mag + 2 * u * np.abs(out)
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * mag * (1 + rel) + 2.0 ** -8 * (np.abs(out) + tol + 2.0 ** -8 * mag)
    return tol + 1e-37, weight + (2 * n + 4) * u + 4 * u * np.abs(np.where(np.isfinite(lse), lse, 0.0))
