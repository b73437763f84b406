"""Sizes that a user cache is refused for, on the host."""
import ctypes as C

import pytest

from paper_2511_12934_amd import binding as B


@pytest.mark.parametrize("max_len,page_len,heads,word", [(2 ** 30 + 1, 1024, 1, "max_len"), (2 ** 31 - 1, 1024, 1, "max_len"), (2 ** 28 + 1, 32, 1, "pages of a sequence"),
                                                         (4096, 1024, 2048, "bytes")])
def test_larger_caches_than_row_numbers_and_grids_reach_are_refused(max_len, page_len, heads, word):
    lib = B.load()
    cfg = B.aif_cache_config(B.AIF_BF16, heads, heads, 256, 0.0, page_len, 4, 1, max_len, 1, 1)
    h = C.c_void_p()
    assert lib.aif_cache_init(C.byref(cfg), C.c_void_p(1 << 20), C.byref(h)) == B.AIF_ESHAPE
    assert word in lib.aif_cache_last_error(None).decode() and not h.value


def test_the_largest_page():
    shape = dict(dtype=B.AIF_BF16, d_head=256, page_len=1024)
    assert B.cache_page_bytes(n_heads=1927, n_kv_heads=1927, **shape) <= 2 ** 29
    with pytest.raises(B.AifError, match="bytes"):
        B.cache_page_bytes(n_heads=1928, n_kv_heads=1928, **shape)
