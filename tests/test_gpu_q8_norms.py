"""8-bit products against 64 bits as a whole (q8_norms.py): sums in too few bits and results a little too large or small lie far below what single values may be off."""
import numpy as np
import pytest

import q8_norms as norms
from paper_2511_12934_amd import binding as B
from test_gpu_q8 import Held, ctx, dev, held, host, repeated, rows_of, say, torch  # noqa: F401  (ctx and torch are fixtures)

pytestmark = pytest.mark.gpu

# rows, k, n: blocks of 16, 32 and 64 rows, small and large tiles; contractions where single values' bounds are wide
SIZES = [(1, 4096, 4096), (64, 1000, 2048), (200, 2048, 2048), (2000, 1152, 1096), (6000, 2048, 520), (20011, 2048, 1096)]
SOME = 60           # rows held against 64 bits


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_norms(torch, ctx, dtype, m, k, n):  # noqa: F811
    rng = np.random.default_rng(m + 3 * k + n)
    some = min(m, SOME)
    base, a64 = held(torch, rng, some, k)
    a = repeated(torch, rng, base, np.arange(m) % some)
    w, w64 = held(torch, rng, n, k, 128)
    up, up64 = held(torch, rng, n, k, 128)
    shift = int(round(np.log2(k) / 2))
    for q in (w, up):
        q.wide_scales[1:-1, :q.across] -= shift
    w64, up64 = w64 / 2.0 ** shift, up64 / 2.0 ** shift
    bias, res = rows_of(rng, 1, n, dtype)[0], rows_of(rng, some, n, dtype)
    for what in ("plain", "bias relu residual", "gate", "gate residual"):
        say(f"norms {dtype} {m} x {k} x {n} {what}")
        args, want = {}, {}
        if "bias" in what:
            args.update(bias=dev(torch, bias[None], dtype)[0], relu=True)
            want.update(bias=bias.astype(np.float64), relu=True)
        if "gate" in what:
            args["up"], want["up"] = up.q, up64
        if "residual" in what:
            args["residual"], want["residual"] = dev(torch, res[np.arange(m) % some], dtype), res.astype(np.float64)
        y64, d = norms.linear(a64, w64, dtype, **want)
        out, q = dev(torch, np.zeros((m, n)), dtype), Held(torch, m, n)
        ctx.aif_q8_linear(B.Q8Linear(a.q, w.q, out, **args))
        ctx.aif_q8_linear(B.Q8Linear(a.q, w.q, q.q, dtype=B.AIF_F32 if dtype == "f32" else B.AIF_BF16, **args))
        last = slice(m - m % some - some, m - m % some) if m % some else slice(m - some, m)     # the last whole turn of the rows
        codes, scales = q.q.codes.cpu().numpy(), q.q.scales.cpu().numpy()
        for at in (slice(0, some), last):
            norms.check_rows(host(out[at]), y64, d, dtype, what)
            norms.check_held(codes[at], scales[at], y64, d, what + " codes")
