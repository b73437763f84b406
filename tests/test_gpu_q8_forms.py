"""Products of few 8-bit rows whose blocks take 32 of them, which test_gpu_q8.py's sizes do not reach, against 64 bits as there."""
import pytest

import test_gpu_q8 as base
from test_gpu_q8 import ctx, torch  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu

SHAPES = [  # rows, k, n: with and without rows left over, columns of k left over, columns of the last strip
    (33, 136, 2040), (64, 1000, 2048), (100, 1152, 1024), (17, 128, 2600), (32, 4096, 4096), (47, 2064, 2000), (96, 8, 1360), (130, 904, 808)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_linear(torch, ctx, dtype, m, k, n):  # noqa: F811
    base.test_linear(torch, ctx, dtype, m, k, n)
