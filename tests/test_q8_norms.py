"""What 8-bit products are held to as a whole (q8_norms.py), without a GPU: right sums pass, sums in too few bits and results a little too large do not."""
import numpy as np
import pytest

import q8_norms as norms
import q8_reference as ref

SIZES = [(79, 640, 1000), (80, 1152, 1100), (60, 2048, 1024)]


def inputs(m, k, n):
    rng = np.random.default_rng(m + k + n)
    make = lambda r, block: ref.values(*ref.hold(rng.standard_normal((r, k)) * np.exp(0.7 * rng.standard_normal(k)) * np.exp(rng.standard_normal((r, 1))), block), block)  # noqa: E731
    return make(m, 1), make(n, 128) / 2.0 ** round(np.log2(k) / 2)


def truncated(x, step):
    return np.trunc(x / step) * step


def summed(a, w, how):
    """Sums as a kernel might have them: fp32 throughout; fp32 between groups of eight that are cut off 13 places below their largest; and rounded to bf16 after each 128 columns."""
    m, k = a.shape
    out = np.zeros((m, w.shape[0]), np.float32)
    for g in range(k // 8):
        p = a[:, None, g * 8:g * 8 + 8] * w[None, :, g * 8:g * 8 + 8]
        if how == "cut off":
            p = truncated(p, 2.0 ** (np.floor(np.log2(np.maximum(np.abs(p).max(2, keepdims=True), 2.0 ** -100))) - 13))
        out += p.sum(2).astype(np.float32)
        if how == "bf16 sums" and g % 16 == 15:
            out = norms.round_bf16(out.astype(np.float64))[0].astype(np.float32)
    return out.astype(np.float64)


def left(z, dtype):
    return z.astype(np.float32) if dtype == "f32" else norms.round_bf16(z)[0]


@pytest.mark.parametrize("m,k,n", SIZES)
def test_what_passes_and_what_does_not(m, k, n):
    a, w = inputs(m, k, n)
    sums = {how: summed(a, w, how) for how in ("fp32", "cut off", "bf16 sums")}
    for dtype in ("f32", "bf16"):
        want, d = norms.linear(a, w, dtype)
        for how, z in [*sums.items(), ("a little large", sums["fp32"] * 1.004)]:
            right = how == "fp32" or (how == "cut off" and dtype == "bf16")
            for check in (lambda: norms.check_rows(left(z, dtype), want, d, dtype, how), lambda: norms.check_held(*ref.hold(z), want, d, how)):
                if right:
                    check()
                else:
                    with pytest.raises(AssertionError, match="is allowed|are expected"):
                        check()
