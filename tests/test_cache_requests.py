"""Requests of the user cache on the host: which tensors they take, whatever their number of rows."""
import pytest

from paper_2511_12934_amd import binding as B


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def _requests(seq, bad, good):
    """Every tensor of every request, one at a time the bad one."""
    return [lambda: B.CacheAppend(seq, bad, good), lambda: B.CacheAppend(seq, good, bad), lambda: B.CacheQuery(seq, bad, good),
            lambda: B.CacheQuery(seq, good, bad), lambda: B.CacheRead(seq, bad, good), lambda: B.CacheRead(seq, good, bad),
            lambda: B.CacheRead(seq, bad, None), lambda: B.CacheRead(seq, None, bad)]


@pytest.mark.parametrize("n", (1, 2, 7))
def test_rows_whose_features_lie_apart_are_refused(torch, n):
    heads, d = 4, 16
    good = torch.zeros(n, heads, d)
    fused = torch.zeros(n, heads, 2 * d)
    for bad in (*fused.chunk(2, -1), fused[:, :, ::2], torch.zeros(n, d, heads).transpose(1, 2), torch.zeros(n, 1, d).expand(n, heads, d),
                torch.zeros(n, heads, 1).expand(n, heads, d)):
        for make in _requests(0, bad, good):
            with pytest.raises(ValueError, match="contiguous"):
                make()


@pytest.mark.parametrize("shape", ((30, 64), (2, 4, 16)))
def test_one_row_that_stands_for_many_is_refused(torch, shape):
    good = torch.zeros(shape)
    for bad in (torch.zeros(1, *shape[1:]).expand(shape), torch.zeros(500).as_strided(shape, (8, *good.stride()[1:]))):
        for make in _requests(0, bad, good):
            with pytest.raises(ValueError, match="overlap"):
                make()


def test_rows_that_are_taken(torch):
    """One row of a wider tensor, rows of a step, heads of one that share their features' order, no rows at all."""
    wide = torch.zeros(6, 3, 40)
    for t, stride in ((wide[2:3, 1], 0), (wide[:, 1], 120), (wide[::3, :2], 360), (wide[:1, :2], 0), (wide[:, :1].transpose(0, 1)[:, 2:4], None),
                      (torch.zeros(1, 4, 16).expand(1, 4, 16), 0), (wide[:0], 0), (torch.zeros(1, 0, 16).expand(5, 0, 16), 0)):
        if stride is None:
            t = t[0]                        # [2, 40], rows 120 apart
            stride = 120
        width = t[0].numel() if t.shape[0] else 0
        assert B._row_stride(t, width) == stride
        assert B.CacheAppend(0, t, t).strides == B.CacheQuery(0, t, t).strides == B.CacheRead(0, t, t).strides == (stride, stride)
