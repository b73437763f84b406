"""Every code under every scale that the calls write, through a product that leaves each as it is (include/aif_q8.h: what a matrix holds stands exactly in bf16 and in fp32)."""
import numpy as np
import pytest

import q8_reference as ref
from paper_2511_12934_amd import binding as B
from test_gpu_q8 import Held, ctx, dev, host, say, torch  # noqa: F401  (ctx and torch are fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("side", ["a", "w"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("times", [1, 130])
def test_products_of_every_code_and_scale(torch, ctx, dtype, times, side):  # noqa: F811
    """a (or w) holds every code under scale bytes 10..246 (under 247 the largest are beyond fp32), the other side a one where column and row are alike."""
    say(f"every code of {side}, {dtype}, {times} times")
    blocks = 237
    codes = np.arange(256, dtype=np.uint8)
    codes[codes & 127 == 127] = 0
    one = np.zeros((256, 256), np.uint8)
    np.fill_diagonal(one, 0x38)
    few = lambda r, b: np.full((r, 4), b, np.uint8)  # noqa: E731
    if side == "a":                             # a row to a scale
        bytes_ = np.repeat(np.tile(np.arange(10, 247, dtype=np.uint8), times)[:, None], 4, 1)
        a, w, w_scales = np.tile(codes, (blocks * times, 1)), one, few(2, 127)
        want = ref.values(a[:blocks], bytes_[:blocks])
        a_scales = bytes_
    else:                                       # 128 rows of the layer to a scale: half of the codes each, over and over
        w = np.zeros((blocks * 128, 256), np.uint8)
        w[np.arange(blocks * 128), np.arange(blocks * 128) % 256] = codes[np.arange(blocks * 128) % 256]
        w_scales = np.repeat(np.arange(10, 247, dtype=np.uint8)[:, None], 4, 1)
        a, a_scales = np.tile(one, (max(times // 16, 1), 1)), few(256 * max(times // 16, 1), 127)
        want = ref.values(w, w_scales, 128).T
    out = dev(torch, np.zeros((a.shape[0], w.shape[0])), dtype)
    ctx.aif_q8_linear(B.Q8Linear(Held(torch, *a.shape, codes=a, scales=a_scales).q, Held(torch, *w.shape, 128, codes=w, scales=w_scales).q, out))
    got = out.view(-1, *want.shape)
    assert all(torch.equal(got[i], got[0]) for i in range(got.shape[0]))
    assert np.array_equal(host(got[0]), want)
