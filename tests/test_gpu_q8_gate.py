"""The gate of an 8-bit layer, SiLU(z) * u, over the whole range in which it is a normal number (include/aif_q8.h)."""
import numpy as np
import pytest

import q8_reference as ref
from paper_2511_12934_amd import binding as B
from test_gpu_q8 import Held, ctx, dev, host, say, torch  # noqa: F401  (ctx and torch are fixtures)

pytestmark = pytest.mark.gpu
# z is the sum of two codes, of columns that no instruction adds in less than fp32, so that it is exact and all that is off is the gate's own: the exponential's
# argument is rounded once (half a step of at most |z| log2 e + 8, times ln 2: (|z| + 5.6) 2^-24 of the exponential), the exponential and the reciprocal are off by 2^-23
# each, an addition and at most three products by 2^-24 each: (|z| / 2 + 6.8) 2^-23.  The reciprocal is brought back by 2^-8 (fp32: by 2^-4, z by the rest) to where
# steps are 2^-149, half a step of which goes times z (fp32: times z 2^-4).  What is itself below 2^-126 counts as nothing.
U23 = 2.0 ** -23


def allowed(dtype, z, s):
    own = (np.abs(z) / 2 + 6.8) * U23 * np.abs(s) + np.abs(z) * (2.0 ** -154 if dtype == "f32" else 2.0 ** -150)
    return np.where(np.abs(s) < 2.0 ** -126, 2.0 ** -126, own)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [40, 900, 20000])
def test_gate_far_from_zero(torch, ctx, dtype, rows):  # noqa: F811
    say(f"gate {dtype} {rows} rows")
    n, k = 264, 24
    hi = np.concatenate([np.arange(64, 121, 8.0), np.arange(32, 64, 4.0), np.arange(0, 32, 2.0)])
    hi = np.concatenate([hi, -hi])
    lo = np.arange(-7.5, 8.0, 0.5)
    grid = np.array([(x, y) for x in hi for y in lo])
    rng = np.random.default_rng(rows)
    pairs = grid[rng.integers(len(grid), size=rows)]
    pairs[:8] = [(-88, -0.5), (-88, -1.5), (-88, -3.0), (-88, 1.0), (-88, 0.5), (-96, 4.5), (-120, -7.5), (120, 7.5)]
    code = {v: i for i, v in reversed(list(enumerate(ref.CODES))) if v == v}
    a = np.zeros((rows, k), np.uint8)
    a[:, 0], a[:, 8], a[:, 16] = [code[x] for x in pairs[:, 0]], [code[y] for y in pairs[:, 1]], code[1.0]
    w, up = np.zeros((n, k), np.uint8), np.zeros((n, k), np.uint8)
    w[:, 0] = w[:, 8] = code[1.0]
    up[:, 16] = 8 * rng.integers(3, 12, n) + rng.integers(0, 8, n) + 128 * rng.integers(0, 2, n)
    scale = lambda r, e: np.repeat(np.full((r, 1), 127 + e, np.uint8), 4, 1)  # noqa: E731
    up_scales = np.stack([scale(1, e)[0] for e in (100, 0, 60)])            # z * u from 2^-40 on, below, and of ordinary size: a block of columns each
    z = pairs.sum(1)[:, None]
    assert z.min() < -100 and z.max() > 100
    s, u = ref.silu(z), ref.values(up, up_scales, 128)[:, 16][None]
    want, off = s * u, allowed(dtype, z, s) * np.abs(u)
    d_a, d_w, d_up = Held(torch, rows, k, codes=a, scales=scale(rows, 0)), Held(torch, n, k, 128, codes=w, scales=scale(3, 0)), Held(torch, n, k, 128, codes=up, scales=up_scales)
    out = dev(torch, np.zeros((rows, n)), dtype)
    ctx.aif_q8_linear(B.Q8Linear(d_a.q, d_w.q, out, up=d_up.q))
    ref.check_rows(host(out), want, off, dtype, "rows")
    q = Held(torch, rows, n)
    ctx.aif_q8_linear(B.Q8Linear(d_a.q, d_w.q, q.q, up=d_up.q, dtype=B.AIF_F32 if dtype == "f32" else B.AIF_BF16))
    codes, scales = q.host()
    ref.check_held(codes[:300], scales[:300], want[:300], off[:300], what="codes")
    res = dev(torch, np.where(want == 0, 1.0, 0.0), dtype)
    ctx.aif_q8_linear(B.Q8Linear(d_a.q, d_w.q, res, up=d_up.q, residual=res))
    ref.check_rows(host(res), np.where(want == 0, 1.0, want), off, dtype, "over a residual")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [3, 20000])
def test_gate_of_the_largest_numbers(torch, ctx, dtype, rows):  # noqa: F811
    """z beyond 2^120 either way, and up to an infinity: z * u, nothing, and z / (1 + exp(-z)) as it stands."""
    say(f"largest gate {dtype} {rows} rows")
    k, n = 8, 128
    a, w, up = np.zeros((rows, k), np.uint8), np.zeros((n, k), np.uint8), np.zeros((n, k), np.uint8)
    a[:, 0], a[:, 1] = 0x38, 0x38
    a[1::3, 0] = 0xB8                                                       # -1
    w[:, 0], up[:, 1] = 0x78, 0x38                                          # 256, 1
    scales = lambda r, b: np.full((r, 4), b, np.uint8)  # noqa: E731
    d_a, d_up = Held(torch, rows, k, codes=a, scales=scales(rows, 127)), Held(torch, n, k, 128, codes=up, scales=scales(1, 107))
    for byte in (127 + 112, 127 + 119):                                     # z = +- 2^120, +- 2^127
        out = dev(torch, np.zeros((rows, n)), dtype)
        d_w = Held(torch, n, k, 128, codes=w, scales=scales(1, byte))
        ctx.aif_q8_linear(B.Q8Linear(d_a.q, d_w.q, out, up=d_up.q))
        want = np.where(np.arange(rows) % 3 == 1, 0.0, 2.0 ** (byte - 127 + 8 - 20))
        assert np.array_equal(host(out), np.repeat(want[:, None], n, 1))
