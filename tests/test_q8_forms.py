"""Which kernel and tile the sizes of an 8-bit product choose (csrc/k_q8_form.h), without a GPU."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2511_12934_amd import build


@pytest.fixture(scope="module")
def form(tmp_path_factory):
    """(rows, k, n, end) -> (few, rows of a tile, its columns); end: words of relu, gate, bias, codes, residual, f32."""
    so = str(tmp_path_factory.mktemp("q8_form") / "form.so")
    subprocess.check_call([build.HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", build.CSRC,
                           os.path.join(os.path.dirname(__file__), "q8_form_host.cpp"), "-o", so])
    lib = C.CDLL(so)

    def of(m, k, n, end="", n_cu=256):
        out = (C.c_int * 3)()
        lib.form(m, k, n, 2 if "gate" in end else int("relu" in end), int("f32" in end), int("codes" in end), int("residual" in end), int("bias" in end), n_cu, out)
        return bool(out[0]), out[1], out[2]
    return of


# Products of bf16 measured with tiles of 256 by 256 and of 128 by 128 in turn, us: rows, columns, end, {columns of k: (large, small)}
MEASURED = [
    (10000, 1024, "", {256: (12.2, 10.8), 512: (14.5, 13.3), 1024: (18.8, 18.7), 2048: (27.5, 30.4), 4096: (44.9, 55.8), 8192: (85.1, 132.1)}),
    (10000, 1024, "codes", {256: (16.7, 14.1), 512: (18.7, 16.9), 1024: (23.0, 22.2), 2048: (31.8, 33.9), 4096: (49.4, 59.5), 8192: (88.1, 131.9)}),
    (6144, 1536, "", {256: (12.7, 10.9), 512: (14.9, 13.6), 1024: (19.2, 18.9), 2048: (28.0, 30.6), 4096: (45.4, 55.8), 8192: (79.9, 106.9)}),
    (2816, 4096, "codes", {256: (17.1, 14.4), 512: (19.2, 17.2), 1024: (23.5, 22.3), 2048: (32.3, 34.0), 4096: (50.2, 59.5), 8192: (85.6, 110.6)}),
    (8192, 1536, "codes", {256: (17.0, 14.5), 512: (19.1, 17.2), 1024: (23.4, 22.4), 2048: (32.3, 34.5), 4096: (50.9, 60.9), 8192: (89.4, 113.9)}),
    (8192, 1024, "", {128: (10.7, 8.0), 1024: (18.6, 14.2), 4096: (45.0, 39.8)}),
    (16384, 1024, "", {128: (11.7, 11.4), 1024: (20.3, 23.9), 4096: (57.8, 85.5)}),
    (16384, 1024, "residual", {128: (18.4, 15.8), 512: (22.1, 20.9), 1024: (27.0, 27.8), 4096: (67.6, 93.5)}),
    (19200, 1024, "", {128: (16.8, 12.4), 512: (23.7, 19.2), 1024: (32.4, 29.4), 2048: (51.6, 49.7)}),
    (24576, 1024, "residual", {128: (40.0, 30.0), 512: (47.2, 39.1), 1024: (55.4, 52.2), 4096: (117.2, 136.9)}),
    (24576, 1024, "", {128: (17.0, 14.8), 512: (24.0, 22.4), 1024: (33.1, 34.7), 2048: (57.2, 70.6), 4096: (100.3, 128.4)}),
    (25600, 1024, "codes", {128: (27.2, 22.8), 512: (33.9, 30.2), 1024: (42.6, 42.0), 2048: (61.6, 69.3), 4096: (107.3, 151.5)}),
    (40960, 1024, "residual", {128: (56.1, 46.2), 256: (60.1, 50.7), 512: (67.3, 60.2), 2048: (112.6, 129.3)}),
    (65536, 1024, "", {128: (32.3, 47.1), 1024: (79.5, 118.1), 4096: (225.2, 334.9)}),
    (65536, 1024, "codes", {128: (49.8, 45.4), 256: (55.3, 51.3), 512: (69.1, 75.8), 4096: (235.6, 334.0)}),
    (25222, 872, "bias", {656: (36.6, 32.3)}),
    (10168, 1752, "bias", {1440: (49.4, 44.1)}),
    (37255, 1128, "bias", {144: (37.5, 32.5)}),
    (39434, 736, "bias", {1368: (53.2, 63.7)}),
    (54347, 552, "bias", {3888: (155.8, 186.1)}),
    (100000, 256, "residual", {128: (39.8, 32.9), 256: (42.6, 37.2), 1024: (59.0, 64.2), 2048: (81.5, 101.0)}),
]


@pytest.mark.parametrize("m,n,end,times", MEASURED, ids=lambda v: str(v) if not isinstance(v, dict) else "")
def test_large_or_small_tiles(form, m, n, end, times):
    """The chosen tiles took at most an eighth more than the others, whatever the contraction: for few columns of it small ones, for many large ones."""
    for k, (large, small) in times.items():
        few, rows, cols = form(m, k, n, end)
        assert not few and (rows, cols) in ((256, 256), (128, 128))
        took = large if rows == 256 else small
        assert took <= 1.125 * min(large, small), (m, k, n, end, rows, large, small)


def test_every_form_is_compared_with_64_bits(form):
    """Each kernel and tile is reached, with each type and with and without a gate, by the sizes that test_gpu_q8.py and test_gpu_q8_forms.py hold against 64 bits."""
    import test_gpu_q8 as base
    import test_gpu_q8_forms as more
    many = next(m.args[1] for m in base.test_linear_of_many_rows.pytestmark if m.args[0] == "m,n,k")
    shapes = base.SHAPES + more.SHAPES + [(m, k, n) for m, n, k in many]
    for dtype in ("f32", ""):
        for end in ("", "bias relu residual", "gate", "gate residual"):
            for where in ("", "codes"):
                got = {form(m, k, n, f"{end} {where} {dtype}") for m, k, n in shapes}
                want = {(True, 16, 128)} if where else {(True, 16, 16), (True, 32, 16), (True, 64, 16)}
                want.add((False, 128, 128))
                if not dtype:
                    want.add((False, 256, 128) if "gate" in end else (False, 256, 256))
                assert got == want, (dtype, end, where, got ^ want)
    # blocks of 32 rows: the other file's alone
    assert {form(*s, end) for s in more.SHAPES for end in ("", "f32", "gate", "gate residual f32")} == {(True, 32, 16)}
    assert not any(form(*s, end)[1] == 32 for s in shapes[:len(base.SHAPES)] for end in ("", "f32"))
