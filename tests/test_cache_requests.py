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


class Calls:
    """The library's sizes, and calls that only count."""

    def __init__(self, real):
        self.aif_cache_page_bytes, self.seen = real.aif_cache_page_bytes, []

    def __getattr__(self, name):
        def call(*args):
            self.seen.append(name)
            return B.AIF_OK
        return call


class Pool:
    """A pool on the requests' device as far as the binding looks at it."""

    def __init__(self, device, pages=4, cuda=True, close=True):
        self.device, self.pages, self.is_cuda, self.close = device, pages, cuda, close

    def numel(self):
        return self.pages * B.cache_page_bytes(**SHAPE)

    def element_size(self):
        return 1

    def is_contiguous(self):
        return self.close

    def data_ptr(self):
        return 64


SHAPE = dict(dtype=B.AIF_BF16, n_heads=4, n_kv_heads=2, d_head=16, page_len=32)


@pytest.fixture
def lib(monkeypatch):
    calls = Calls(B.load())
    monkeypatch.setattr(B, "load", lambda: calls)
    monkeypatch.setattr(B, "_stream", lambda: None)
    monkeypatch.setattr(B, "_current_device", lambda: None)
    return calls


def _context(torch, lib, **kw):
    return B.CacheContext(pool=kw.pop("pool", Pool(torch.device("cpu"))), max_seqs=4, max_len=100, max_requests=8, max_queries=8, **{**SHAPE, **kw})


@pytest.mark.parametrize("beforehand", (False, True))
def test_requests_packed_beforehand_are_held_against_the_context_too(torch, lib, beforehand):
    ctx = _context(torch, lib)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    q, lse = bf(3, 4, 16), torch.zeros(3, 4)
    append = (ctx.aif_cache_append, B.pack_cache_appends)
    attend = (ctx.aif_cache_attend, B.pack_cache_queries)
    reads = (ctx.aif_cache_read, B.pack_cache_reads)
    fine = [(append, B.CacheAppend(0, bf(3, 2, 16), bf(3, 2, 16))),
            (attend, B.CacheQuery(0, q, q, lse=lse, positions=torch.zeros(3, dtype=torch.int32))), (attend, B.CacheQuery(0, q[:0], q[:0])),
            (attend, B.CacheQuery(0, q[:1], q[:1], lse=lse[:1])), (reads, B.CacheRead(0, None, bf(3, 32))), (reads, B.CacheRead(0, bf(3, 32), None))]
    bad = [(append, "keys has rows of 32 torch.float32", B.CacheAppend(0, torch.zeros(3, 32), torch.zeros(3, 32))),
           (append, "vals has rows of 32 torch.float32", B.CacheAppend(0, bf(3, 32), torch.zeros(3, 32))),
           (append, "keys has rows of 64", B.CacheAppend(0, bf(3, 64), bf(3, 64))),
           (append, "keys has rows of 32 torch.bfloat16 on meta", B.CacheAppend(0, bf(3, 32).to("meta"), bf(3, 32))),
           (attend, "q has rows of 32", B.CacheQuery(0, bf(3, 2, 16), bf(3, 2, 16))),
           (attend, "out has rows of 64 torch.float32", B.CacheQuery(0, q, q.float())),
           (attend, "lse is", B.CacheQuery(0, q, q, lse=torch.zeros(3, 2))), (attend, "lse is", B.CacheQuery(0, q, q, lse=torch.zeros(3, 0))), (attend, "lse is", B.CacheQuery(0, q, q, lse=lse.double())),
           (attend, "positions are int32", B.CacheQuery(0, q, q, positions=torch.zeros(3, dtype=torch.int64))),
           (reads, "keys_out has rows of 16", B.CacheRead(0, bf(3, 16), None)), (reads, "vals_out has rows of 32 torch.float16", B.CacheRead(0, None, bf(3, 32).half()))]
    lib.seen.clear()
    for (call, pack), r in fine:
        many = [r] * 3
        call(many, packed=pack(many) if beforehand else None)
        call(many[:2], **({"packed": pack(many)} if beforehand else {}))
    assert len(lib.seen) == 2 * len(fine)
    for (call, pack), word, r in bad:
        many = [x for (c, _), x in fine if c == call][:1] * ("meta" not in word) + [r]       # (beside the CPU, this context's device, meta goes for none)
        for _ in range(2):
            with pytest.raises(ValueError, match=f"request {len(many) - 1}: {word}"):
                call(many, packed=pack(many) if beforehand else None)
    assert len(lib.seen) == 2 * len(fine)


def test_a_packed_array_serves_the_contexts_that_it_fits(torch, lib):
    a, b = _context(torch, lib), _context(torch, lib, n_kv_heads=4)
    rows = [B.CacheAppend(0, torch.zeros(3, 32, dtype=torch.bfloat16), torch.zeros(3, 32, dtype=torch.bfloat16))]
    packed = B.pack_cache_appends(rows)
    for _ in range(2):
        a.aif_cache_append(rows, packed=packed)
        with pytest.raises(ValueError, match="rows of 32"):
            b.aif_cache_append(rows, packed=packed)


def test_more_requests_than_were_packed_are_refused(torch, lib):
    ctx = _context(torch, lib)
    x = torch.zeros(3, 32, dtype=torch.bfloat16)
    r = B.CacheAppend(0, x, x)
    lib.seen.clear()
    for packed in (B.pack_cache_appends([r]), (B.aif_cache_append_req * 1)()):
        with pytest.raises(ValueError, match="2 requests"):
            ctx.aif_cache_append([r, r], packed=packed)
    with pytest.raises(ValueError, match="1 requests"):
        ctx.aif_cache_append([r], packed=B.pack_cache_appends([]))
    assert not lib.seen


def test_pools_refused(torch, lib):
    cpu = torch.device("cpu")
    for pool in (Pool(cpu, cuda=False), Pool(cpu, close=False)):
        with pytest.raises(ValueError, match="pool"):
            _context(torch, lib, pool=pool)
        with pytest.raises(ValueError, match="pool"):
            _context(torch, lib).aif_cache_swap_pool(pool)
    with pytest.raises(ValueError, match="pool"):
        _context(torch, lib).aif_cache_swap_pool(Pool(torch.device("cuda", 1)))


@pytest.mark.parametrize("number", (2 ** 31, 2 ** 32, 2 ** 32 + 1, -2 ** 31 - 1))
def test_numbers_beyond_32_bits_are_refused(torch, lib, number):
    """(A C field keeps their low 32 bits without a word: 2^32 + 1 would be sequence 1, a window of 2^32 none.)"""
    ctx = _context(torch, lib)
    x = torch.zeros(3, 4, 16, dtype=torch.bfloat16)
    lib.seen.clear()
    for f in (lambda: B.CacheAppend(number, x, x), lambda: B.CacheQuery(number, x, x), lambda: B.CacheQuery(0, x, x, sinks=number),
              lambda: B.CacheQuery(0, x, x, window=number), lambda: B.CacheRead(number, x, x), lambda: B.CacheRead(0, x, x, first=number),
              lambda: B.cache_ids([0, number]), lambda: ctx.aif_cache_free([number]), lambda: ctx.aif_cache_fork([0], [number]),
              lambda: ctx.aif_cache_truncate(number, 0), lambda: ctx.aif_cache_truncate(0, number), lambda: ctx.aif_cache_trim([0], number, 1),
              lambda: ctx.aif_cache_trim([0], 0, number), lambda: ctx.aif_cache_swap_pool(Pool(torch.device("cpu")), number),
              lambda: _context(torch, lib, page_len=number), lambda: B.CacheContext(pool=Pool(torch.device("cpu")), max_seqs=4, max_len=number, max_requests=8, **SHAPE),
              lambda: B.CacheContext(pool=Pool(torch.device("cpu")), max_seqs=number, max_len=9, max_requests=8, **SHAPE)):
        with pytest.raises(ValueError, match="32 bits|the pool holds"):
            f()
    assert set(lib.seen) <= {"aif_cache_destroy"}
    lib.aif_cache_len = lambda h, seq: seq if seq >= 0 else -1
    assert ctx.aif_cache_len(number) == -1 and ctx.aif_cache_len(3) == 3        # "outside the context"
    assert list(B.cache_ids([5, 2 ** 31 - 1, -1])) == [5, 2 ** 31 - 1, -1] and B.CacheQuery(0, x, x, window=2 ** 31 - 1).window == 2 ** 31 - 1


@pytest.mark.parametrize("scale,status", ((2.36e38, B.AIF_EINVAL), (3.4e38, B.AIF_EINVAL), (-1e-30, B.AIF_EINVAL)))
def test_scales_that_no_score_in_powers_of_two_has_are_refused(scale, status):
    """scale / ln 2 has to be a number."""
    import ctypes as C
    cfg = B.aif_cache_config(B.AIF_BF16, 4, 2, 16, scale, 32, 4, 2, 100, 2, 1)
    out = C.c_void_p()
    assert B.load().aif_cache_init(C.byref(cfg), 64, C.byref(out)) == status and not out.value
    assert b"scale" in B.load().aif_cache_last_error(None)
