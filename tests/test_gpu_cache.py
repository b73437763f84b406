"""The user cache on the GPU through the C ABI (include/aif_cache.h) against its 64-bit reference."""
import ctypes as C

import numpy as np
import pytest

import cache_reference as ref
from paper_2511_12934_amd import binding as B
from paper_2511_12934_amd import workloads as wl

pytestmark = pytest.mark.gpu


def _say(msg):
    print(f"[case] {msg}", flush=True)


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def dev(torch, x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(torch.float32 if dtype == "f32" else torch.bfloat16)


def host(t):
    return t.detach().float().cpu().numpy()


def make(torch, dtype, heads, kv, d, pl=64, pages=64, seqs=8, longest=4000, requests=16, queries=4096, fill=0xff, **kw):
    """A cache over a pool whose bytes are all `fill`: what nobody wrote reads as NaN."""
    shape = dict(dtype=B.AIF_F32 if dtype == "f32" else B.AIF_BF16, n_heads=heads, n_kv_heads=kv, d_head=d, page_len=pl)
    pool = torch.full((pages * B.cache_page_bytes(**shape),), fill, dtype=torch.uint8, device="cuda")
    return B.CacheContext(pool=pool, max_seqs=seqs, max_len=longest, max_requests=requests, max_queries=queries, **shape, **kw)


def rows(rng, n, kv, d, dtype, spread=1.0):
    x = rng.standard_normal((n, kv, d)) * np.exp(0.7 * rng.standard_normal((kv, d))) * spread
    return wl.round_storage(x.astype(np.float32), dtype)


def fill(torch, ctx, dtype, seq, k, v, cuts=()):
    """Appends in pieces."""
    for lo, hi in zip((0, *cuts), (*cuts, len(k))):
        ctx.aif_cache_append([B.CacheAppend(seq, dev(torch, k[lo:hi], dtype), dev(torch, v[lo:hi], dtype))])


def read(torch, ctx, dtype, seq, kv, d, first=0, n=None):
    n = ctx.aif_cache_len(seq) - first if n is None else n
    out = [torch.full((n, kv, d), 7.0, device="cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16) for _ in range(2)]
    ctx.aif_cache_read([B.CacheRead(seq, out[0], out[1], first=first)])
    return host(out[0]), host(out[1])


def check_attend(torch, ctx, dtype, seq, keys, vals, q, *, scale, positions=None, sinks=0, window=0, dropped=(), what="", lse=True):
    """One entry against the reference; keys and vals as appended."""
    n_q, heads, d = q.shape
    dq = dev(torch, q, dtype)
    out = torch.full_like(dq, float("nan"))
    got_lse = torch.full((n_q, heads), float("nan"), device="cuda") if lse else None
    dp = None if positions is None else torch.from_numpy(np.asarray(positions, np.int32)).cuda()
    ctx.aif_cache_attend([B.CacheQuery(seq, dq, out, lse=got_lse, positions=dp, sinks=sinks, window=window)])
    torch.cuda.synchronize()
    compare(dtype, host(out), host(got_lse) if lse else None, q, keys, vals, scale, positions, sinks, window, dropped, what)
    return host(out)


def compare(dtype, out, lse, q, keys, vals, scale, positions=None, sinks=0, window=0, dropped=(), what=""):
    n, (n_q, heads, d) = len(keys), q.shape
    see = ref.sees(n, np.full(n_q, n - 1) if positions is None else positions, sinks, window, dropped)
    want, want_lse, mag, big, top = ref.attend(q, ref.hold(keys), ref.hold(vals), scale, see)
    tol, tol_lse = ref.tolerances(dtype, d, n, want, want_lse, mag, big, top)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(out), nan), f"{what}: NaN in other places"
    err = np.abs(out - want)[~nan]
    assert np.all(err <= tol[~nan]), f"{what}: off by {err.max():.3e}, {(err / tol[~nan]).max():.2f} of the tolerance"
    if lse is not None:
        fine = np.isfinite(want_lse)
        assert np.array_equal(lse[~fine], want_lse[~fine], equal_nan=True), f"{what}: lse"
        assert np.all(np.abs(lse - want_lse)[fine] <= tol_lse[fine]), f"{what}: lse off by {np.abs(lse - want_lse)[fine].max():.3e}"


@pytest.mark.parametrize("dtype,kv,d,pl", [("bf16", 1, 64, 64), ("f32", 2, 32, 32), ("bf16", 3, 128, 96), ("f32", 1, 20, 32), ("bf16", 2, 16, 128),
                                           ("bf16", 1, 200, 64), ("f32", 4, 256, 32), ("bf16", 8, 40, 1024)])
@pytest.mark.parametrize("n", (1, 33, 301))
def test_rows_come_back_as_the_values_they_stand_for(torch, dtype, kv, d, pl, n):
    _say(f"append, read {dtype} kv={kv} d={d} page={pl} n={n}")
    rng = np.random.default_rng(n)
    ctx = make(torch, dtype, kv, kv, d, pl, pages=40)
    k, v = rows(rng, n, kv, d, dtype), rows(rng, n, kv, d, dtype, 1e-3)
    k[n // 2, 0] = 0
    fill(torch, ctx, dtype, 3, k, v, cuts=(n // 3, n // 2))
    gk, gv = read(torch, ctx, dtype, 3, kv, d)
    assert np.array_equal(gk, ref.hold(k)) and np.array_equal(gv, ref.hold(v))
    first = n // 2
    gk, gv = read(torch, ctx, dtype, 3, kv, d, first=first)
    assert np.array_equal(gk, ref.hold(k)[first:]) and np.array_equal(gv, ref.hold(v)[first:])


def test_ties_extremes_and_what_is_not_finite(torch):
    _say("format: ties, largest and smallest numbers, NaN and infinities")
    for dtype in ("f32", "bf16"):
        k = np.zeros((9, 1, 64), np.float32)
        k[0, 0, :9] = [6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.25]
        k[1, 0, :3] = [6.03125, 5, -7]
        k[2, 0, :2] = [3.3895e38, -1]
        k[3, 0, :4] = [1e-38, 6 * 2.0 ** -125, -2.0 ** -126, 2.0 ** -127]
        k[4, 0, 40] = np.nan
        k[5, 0, 3] = np.inf
        k[6, 0, 3] = -np.inf
        k[7, 0, :2] = [4 * 2.0 ** 100, 2.0 ** 98]
        k[8, 0, :] = -0.0
        k = wl.round_storage(k, dtype)
        ctx = make(torch, dtype, 1, 1, 64)
        fill(torch, ctx, dtype, 0, k, k[::-1].copy())
        gk, gv = read(torch, ctx, dtype, 0, 1, 64)
        assert np.array_equal(gk, ref.hold(k), equal_nan=True), dtype
        assert np.array_equal(gv, ref.hold(k[::-1]), equal_nan=True), dtype


SHAPES = [("bf16", 1, 1, 64), ("bf16", 8, 2, 128), ("f32", 1, 1, 32), ("f32", 6, 2, 40), ("bf16", 8, 8, 16), ("bf16", 2, 1, 256), ("f32", 2, 2, 128),
          ("bf16", 3, 1, 96), ("bf16", 16, 1, 192), ("f32", 5, 1, 80), ("f32", 2, 1, 256)]


@pytest.mark.parametrize("dtype,heads,kv,d", SHAPES)
@pytest.mark.parametrize("n,n_q", [(1, 1), (31, 2), (64, 5), (65, 70), (500, 1), (517, 40), (1300, 9)])
def test_attention_over_the_whole_cache(torch, dtype, heads, kv, d, n, n_q):
    _say(f"attend {dtype} heads={heads}/{kv} d={d} n={n} n_q={n_q}")
    rng = np.random.default_rng(n + d)
    ctx = make(torch, dtype, heads, kv, d, 64 if d != 40 else 32, pages=64)
    k, v = rows(rng, n, kv, d, dtype), rows(rng, n, kv, d, dtype)
    fill(torch, ctx, dtype, 1, k, v)
    q = wl.round_storage(rng.standard_normal((n_q, heads, d)).astype(np.float32), dtype)
    check_attend(torch, ctx, dtype, 1, k, v, q, scale=d ** -0.5, what=f"{dtype} {heads}/{kv} {d}")


@pytest.mark.parametrize("dtype,heads,kv,d", [("bf16", 1, 1, 64), ("bf16", 4, 2, 128), ("f32", 3, 1, 40)])
@pytest.mark.parametrize("sinks,window", [(0, 1), (4, 33), (70, 64), (0, 5000), (1, 300), (5000, 2)])
def test_window_and_sinks(torch, dtype, heads, kv, d, sinks, window):
    _say(f"window {window} sinks {sinks} {dtype} heads={heads}/{kv} d={d}")
    rng = np.random.default_rng(sinks + window)
    n, n_q = 777, 90
    ctx = make(torch, dtype, heads, kv, d, 32, pages=64)
    k, v = rows(rng, n, kv, d, dtype), rows(rng, n, kv, d, dtype)
    fill(torch, ctx, dtype, 0, k, v)
    q = wl.round_storage(rng.standard_normal((n_q, heads, d)).astype(np.float32), dtype)
    pos = rng.integers(-3, n + 40, n_q)
    pos[:6] = (-1, 0, n - 1, -2 ** 31, 2 ** 31 - 1, window - 1)
    check_attend(torch, ctx, dtype, 0, k, v, q, scale=d ** -0.5, positions=pos, sinks=sinks, window=window, what="positions")
    check_attend(torch, ctx, dtype, 0, k, v, np.sort(q, 0), scale=d ** -0.5, positions=np.sort(pos), sinks=sinks, window=window, what="sorted positions")
    check_attend(torch, ctx, dtype, 0, k, v, q[:1], scale=d ** -0.5, sinks=sinks, window=window, what="one query")
    check_attend(torch, ctx, dtype, 0, k, v, q, scale=d ** -0.5, sinks=sinks, window=window, what="no positions", lse=False)
    check_attend(torch, ctx, dtype, 0, k, v, q, scale=d ** -0.5, positions=pos, what="no window")


@pytest.mark.parametrize("n_q", (1, 40, 300))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_rows_that_see_nothing_and_sequences_without_rows(torch, dtype, n_q):
    _say(f"empty {dtype} n_q={n_q}")
    rng = np.random.default_rng(7)
    ctx = make(torch, dtype, 4, 2, 64)
    q = wl.round_storage(rng.standard_normal((n_q, 4, 64)).astype(np.float32), dtype)
    empty = np.zeros((0, 2, 64), np.float32)
    out = check_attend(torch, ctx, dtype, 0, empty, empty, q, scale=0.125, what="no rows")
    assert not out.any()
    k, v = rows(rng, 100, 2, 64, dtype), rows(rng, 100, 2, 64, dtype)
    fill(torch, ctx, dtype, 0, k, v)
    pos = np.full(n_q, -1)
    assert not check_attend(torch, ctx, dtype, 0, k, v, q, scale=0.125, positions=pos, what="before the first").any()
    pos[::2] = 5
    check_attend(torch, ctx, dtype, 0, k, v, q, scale=0.125, positions=pos, sinks=3, window=2, what="every other")
    assert not check_attend(torch, ctx, dtype, 0, k, v, q, scale=0.125, positions=np.full(n_q, 500), window=7, what="behind the last").any()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("n_q", (1, 5, 64, 200))
def test_nan_and_infinities_stay_where_they_are_seen(torch, dtype, n_q):
    _say(f"NaN in hidden and seen places, {dtype} n_q={n_q}")
    rng = np.random.default_rng(11)
    n, heads, kv, d = 150, 4, 2, 128
    ctx = make(torch, dtype, heads, kv, d)
    k, v = rows(rng, n, kv, d, dtype), rows(rng, n, kv, d, dtype)
    k[20, 0, 3] = np.nan
    v[21, 1, 70] = np.inf          # one block of 32 features of one head
    v[100, 0, 0] = np.nan
    fill(torch, ctx, dtype, 2, k, v)
    q = wl.round_storage(rng.standard_normal((n_q, heads, d)).astype(np.float32), dtype)
    pos = rng.integers(0, n, n_q)
    pos[0] = 19
    what = dict(scale=d ** -0.5, positions=pos)
    check_attend(torch, ctx, dtype, 2, k, v, q, what="all before", **what)
    check_attend(torch, ctx, dtype, 2, k, v, q, what="window", window=10, **what)
    check_attend(torch, ctx, dtype, 2, k, v, q, what="window and sinks", window=60, sinks=21, **what)


@pytest.mark.parametrize("n_q", (1, 64))
def test_large_and_infinite_scores(torch, n_q):
    _say(f"scores of any size, n_q={n_q}")
    rng = np.random.default_rng(3)
    for dtype in ("f32", "bf16"):
        ctx = make(torch, dtype, 1, 1, 64)
        k, v = rows(rng, 200, 1, 64, dtype), rows(rng, 200, 1, 64, dtype)
        fill(torch, ctx, dtype, 0, k, v)
        q = wl.round_storage((rng.standard_normal((n_q, 1, 64)) * 300).astype(np.float32), dtype)
        check_attend(torch, ctx, dtype, 0, k, v, q, scale=0.125, what="one key takes all")
        check_attend(torch, ctx, dtype, 0, k, v, q * 1e-30, scale=0.125, what="all alike")
        # every score minus infinity: a key of -1 in one place, a query of the largest number there and a scale above 1
        ctx = make(torch, dtype, 1, 1, 64, scale=4.0)
        k2 = np.zeros((70, 1, 64), np.float32)
        k2[:, 0, 5] = -4
        q2 = np.zeros((n_q, 1, 64), np.float32)
        q2[:, 0, 5] = 3e38
        q2 = wl.round_storage(q2, dtype)
        fill(torch, ctx, dtype, 0, k2, v[:70])
        dq = dev(torch, q2, dtype)
        out, lse = torch.full_like(dq, 9.0), torch.zeros((n_q, 1), device="cuda")
        ctx.aif_cache_attend([B.CacheQuery(0, dq, out, lse=lse)])
        assert not host(out).any() and np.all(np.isneginf(host(lse)))


def test_many_entries_of_unlike_lengths_in_one_call(torch):
    _say("ragged entries, the same sequence named more than once, more entries than travel in arguments")
    rng = np.random.default_rng(5)
    heads, kv, d, n_seq = 4, 2, 64, 70
    ctx = make(torch, "bf16", heads, kv, d, pages=400, seqs=n_seq, requests=200)
    lens = [int(x) for x in rng.integers(0, 300, n_seq)]
    lens[0], lens[1], lens[2] = 0, 1, 700
    ks, vs = zip(*[(rows(rng, n, kv, d, "bf16"), rows(rng, n, kv, d, "bf16")) for n in lens])
    ctx.aif_cache_append([B.CacheAppend(s, dev(torch, ks[s], "bf16"), dev(torch, vs[s], "bf16")) for s in range(n_seq)])
    for n_req, most in ((1, 1), (9, 1), (70, 1), (150, 3), (150, 90)):
        asks, keep = [], []
        for r in range(n_req):
            s, n_q = r % n_seq, int(rng.integers(0, most + 1)) if most > 1 else 1
            q = wl.round_storage(rng.standard_normal((n_q, heads, d)).astype(np.float32), "bf16")
            dq = dev(torch, q, "bf16")
            out, lse = torch.full_like(dq, float("nan")), torch.full((n_q, heads), float("nan"), device="cuda")
            w = int(rng.integers(0, 3)) * 50
            asks.append(B.CacheQuery(s, dq, out, lse=lse, window=w, sinks=3))
            keep.append((s, q, out, lse, w))
        ctx.aif_cache_attend(asks)
        torch.cuda.synchronize()
        first = [host(k[2]) for k in keep]
        ctx.aif_cache_attend(asks)
        torch.cuda.synchronize()
        for (s, q, out, lse, w), before in zip(keep, first):
            assert np.array_equal(host(out), before, equal_nan=True)         # the same call, the same bits
            if q.size:
                compare("bf16", host(out), host(lse), q, ks[s], vs[s], d ** -0.5, sinks=3, window=w, what=f"{n_req} entries, sequence {s}")


def test_rows_that_lie_apart_and_neighbours_left_alone(torch):
    _say("strides")
    rng = np.random.default_rng(6)
    heads, kv, d, n, n_q = 4, 2, 64, 130, 50
    for dtype in ("bf16", "f32"):
        ctx = make(torch, dtype, heads, kv, d)
        k, v = rows(rng, n, kv, d, dtype), rows(rng, n, kv, d, dtype)
        both = dev(torch, np.concatenate([k.reshape(n, -1), v.reshape(n, -1)], 1), dtype)         # [n, K | V]
        ctx.aif_cache_append([B.CacheAppend(0, both[:, :kv * d], both[:, kv * d:])])
        q = wl.round_storage(rng.standard_normal((n_q, heads, d)).astype(np.float32), dtype)
        wide = torch.full((2 * n_q, heads * d + 16), 5.0, device="cuda").to(both.dtype)
        wide[::2, 8:-8] = dev(torch, q.reshape(n_q, -1), dtype)
        res = torch.full_like(wide, 3.0)
        ctx.aif_cache_attend([B.CacheQuery(0, wide[::2, 8:-8], res[::2, 8:-8])])
        torch.cuda.synchronize()
        compare(dtype, host(res[::2, 8:-8]).reshape(n_q, heads, d), None, q, k, v, d ** -0.5, what="strided")
        res[::2, 8:-8] = 3.0
        assert torch.all(res == 3.0)
        out = torch.full((2 * n, 3 * kv * d), 3.0, device="cuda").to(both.dtype)
        ctx.aif_cache_read([B.CacheRead(0, out[1::2, kv * d:2 * kv * d], None)])
        assert np.array_equal(host(out[1::2, kv * d:2 * kv * d]).reshape(n, kv, d), ref.hold(k))
        out[1::2, kv * d:2 * kv * d] = 3.0
        assert torch.all(out == 3.0)


def test_branches_share_pages_until_they_are_written(torch):
    _say("fork, append, truncate, copy, trim, compact, swap_pool, free")
    rng = np.random.default_rng(8)
    dtype, heads, kv, d, pl = "bf16", 2, 2, 64, 32
    ctx = make(torch, dtype, heads, kv, d, pl, pages=60, seqs=12)
    k, v = rows(rng, 200, kv, d, dtype), rows(rng, 200, kv, d, dtype)
    q = wl.round_storage(rng.standard_normal((3, heads, d)).astype(np.float32), dtype)
    want = {}

    def put(seqs, n):
        new = {s: (rows(rng, n, kv, d, dtype), rows(rng, n, kv, d, dtype)) for s in seqs}
        ctx.aif_cache_append([B.CacheAppend(s, dev(torch, a, dtype), dev(torch, b, dtype)) for s, (a, b) in new.items()])
        for s, (a, b) in new.items():
            old = want.get(s, (a[:0], b[:0]))
            want[s] = np.concatenate([old[0], a]), np.concatenate([old[1], b])

    def check(dropped={}):
        for s, (a, b) in want.items():
            assert ctx.aif_cache_len(s) == len(a)
            if s not in dropped:
                gk, gv = read(torch, ctx, dtype, s, kv, d)
                assert np.array_equal(gk, ref.hold(a)) and np.array_equal(gv, ref.hold(b)), s
            check_attend(torch, ctx, dtype, s, a, b, q, scale=d ** -0.5, dropped=dropped.get(s, ()), what=f"sequence {s}")

    put((0, 1), 70)                                   # 3 pages each
    ctx.aif_cache_fork([0, 1, 0], [2, 3, 4])
    want[2], want[3], want[4] = want[0], want[1], want[0]
    assert ctx.aif_cache_free_pages() == 54
    check()
    put((0, 2, 4), 5)                                 # all three leave the shared page
    assert ctx.aif_cache_free_pages() == 52           # three new ones, the shared one is nobody's any more
    check()
    ctx.aif_cache_truncate(4, 68)
    want[4] = want[4][0][:68], want[4][1][:68]
    put((4,), 40)
    check()
    ctx.aif_cache_copy([4, 1], [5, 6])
    want[5], want[6] = want[4], want[1]
    put((6,), 100)
    check()
    ctx.aif_cache_free([0, 1, 1, 5])
    del want[0], want[1], want[5]
    used = ctx.aif_cache_compact()
    assert used == 60 - ctx.aif_cache_free_pages()
    check()
    ctx.aif_cache_trim([6, 6], sinks=10, window=40)   # 170 rows: pages 1..3 of 6 go
    drop = {6: ((32, 128),)}
    check(drop)
    ctx.aif_cache_fork([6], [7])
    want[7], drop[7] = want[6], drop[6]
    ctx.aif_cache_copy([6], [8])
    want[8], drop[8] = want[6], drop[6]
    put((6, 7), 3)
    check(drop)
    check_attend(torch, ctx, dtype, 6, *want[6], q, scale=d ** -0.5, sinks=10, window=40, dropped=drop[6], what="window after trim")
    used = ctx.aif_cache_compact()
    page = B.cache_page_bytes(dtype=B.AIF_BF16, n_heads=heads, n_kv_heads=kv, d_head=d, page_len=pl)
    smaller = torch.full(((used + 2) * page,), 0xff, dtype=torch.uint8, device="cuda")
    smaller[:used * page] = ctx._keep[0][:used * page]
    old = ctx._keep[0]
    ctx.aif_cache_swap_pool(smaller)
    old.fill_(0xff)
    assert ctx.aif_cache_free_pages() == 2
    check(drop)
    put((8,), 33)
    check(drop)


def test_refusals_change_nothing(torch):
    _say("refusals")
    rng = np.random.default_rng(9)
    ctx = make(torch, "bf16", 2, 1, 64, 32, pages=6, seqs=4, longest=150, requests=3, queries=8)
    k = rows(rng, 100, 1, 64, "bf16")
    fill(torch, ctx, "bf16", 0, k, k)
    t = dev(torch, k, "bf16")
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    o = torch.zeros_like(q)
    lib, h = ctx._lib, ctx._h

    def no(status, word, f):
        with pytest.raises(B.AifError, match=word) as e:
            f()
        assert e.value.status == status
        assert ctx.aif_cache_len(0) == 100 and ctx.aif_cache_len(1) == 0 and ctx.aif_cache_free_pages() == 2

    app = lambda *a: ctx.aif_cache_append([B.CacheAppend(*x) for x in a])  # noqa: E731
    no(B.AIF_ERANGE, "outside", lambda: app((4, t, t)))
    no(B.AIF_ERANGE, "outside", lambda: app((-1, t, t)))
    no(B.AIF_EINVAL, "twice", lambda: app((1, t[:3], t[:3]), (1, t[:3], t[:3])))
    no(B.AIF_ERANGE, "max_len", lambda: app((0, t[:51], t[:51])))
    no(B.AIF_ERANGE, "free", lambda: app((1, t[:65], t[:65])))
    no(B.AIF_ERANGE, "free", lambda: app((1, t[:33], t[:33]), (2, t[:1], t[:1])))
    no(B.AIF_ERANGE, "entries", lambda: app(*[(i, t[:1], t[:1]) for i in (1, 2, 3, 0)]))
    ask = lambda **kw: ctx.aif_cache_attend([B.CacheQuery(**{"seq": 0, "q": q, "out": o, **kw})])  # noqa: E731
    no(B.AIF_ERANGE, "outside", lambda: ask(seq=9))
    no(B.AIF_EINVAL, "sinks or window", lambda: ask(window=-1))
    no(B.AIF_EINVAL, "sinks or window", lambda: ask(sinks=-1))
    no(B.AIF_ERANGE, "max_queries", lambda: ask(q=torch.cat([q, q, q]), out=torch.cat([o, o, o])))
    rd = lambda first, n: ctx.aif_cache_read([B.CacheRead(0, t[:n].clone(), None, first=first)])  # noqa: E731
    no(B.AIF_ERANGE, "the sequence has 100", lambda: rd(1, 100))
    no(B.AIF_ERANGE, "the sequence has 100", lambda: rd(101, 1))
    no(B.AIF_EINVAL, "negative", lambda: rd(-1, 1))
    no(B.AIF_EINVAL, "not empty", lambda: ctx.aif_cache_fork([0], [0]))
    no(B.AIF_EINVAL, "twice", lambda: ctx.aif_cache_fork([0, 0], [1, 1]))
    no(B.AIF_EINVAL, "source and destination", lambda: ctx.aif_cache_fork([0, 1], [1, 2]))
    no(B.AIF_ERANGE, "free", lambda: ctx.aif_cache_copy([0], [1]))
    no(B.AIF_ERANGE, "outside", lambda: ctx.aif_cache_free([0, 4]))
    no(B.AIF_ERANGE, "length", lambda: ctx.aif_cache_truncate(0, 101))
    no(B.AIF_ERANGE, "length", lambda: ctx.aif_cache_truncate(0, -1))
    no(B.AIF_EINVAL, "trim", lambda: ctx.aif_cache_trim([0], 0, 0))
    no(B.AIF_ERANGE, "in use", lambda: ctx.aif_cache_swap_pool(ctx._keep[0], 3))
    # raw pointers: NULL, odd addresses, odd strides
    for kw, st in ((dict(keys=None), B.AIF_EINVAL), (dict(vals=t.data_ptr() + 8), B.AIF_EINVAL), (dict(key_stride=65), B.AIF_EINVAL),
                   (dict(key_stride=56), B.AIF_EINVAL), (dict(n_rows=-1), B.AIF_EINVAL)):
        r = B.pack_cache_appends([B.CacheAppend(1, t[:2], t[:2])])
        for f, x in kw.items():
            setattr(r[0], f, x)
        assert lib.aif_cache_append(h, r, 1, None) == st, kw
    for kw in (dict(q=None), dict(out=o.data_ptr() + 2), dict(out_stride=120), dict(lse_out=o.data_ptr() + 2), dict(positions=o.data_ptr() + 1), dict(n_q=-1)):
        r = B.pack_cache_queries([B.CacheQuery(0, q, o)])
        for f, x in kw.items():
            setattr(r[0], f, x)
        assert lib.aif_cache_attend(h, r, 1, None) == B.AIF_EINVAL, kw
    assert lib.aif_cache_append(h, None, 1, None) == B.AIF_EINVAL and lib.aif_cache_attend(h, None, -1, None) == B.AIF_EINVAL
    # the binding's own
    with pytest.raises(ValueError, match="rows of"):
        app((1, t.float(), t.float()))
    with pytest.raises(ValueError, match="rows of"):
        ask(q=q[:, :1], out=o[:, :1])
    with pytest.raises(ValueError, match="positions are int32"):
        ask(positions=torch.zeros(4, dtype=torch.int64, device="cuda"))
    ctx.aif_cache_trim([0], 0, 10)
    with pytest.raises(B.AifError, match="dropped"):
        rd(0, 40)
    with pytest.raises(B.AifError, match="dropped"):
        ctx.aif_cache_truncate(0, 40)
    torch.cuda.synchronize()
    gk, _ = read(torch, ctx, "bf16", 0, 1, 64, first=96)
    assert np.array_equal(gk, ref.hold(k)[96:])


def test_calls_under_capture_are_refused_and_do_not_spoil_it(torch):
    _say("capture")
    ctx = make(torch, "bf16", 1, 1, 64)
    x = torch.ones((4, 1, 64), dtype=torch.bfloat16, device="cuda")
    ctx.aif_cache_append([B.CacheAppend(0, x, x)])
    out, y = torch.zeros_like(x), torch.zeros(8, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    calls = (lambda: ctx.aif_cache_append([B.CacheAppend(1, x, x)]), lambda: ctx.aif_cache_attend([B.CacheQuery(0, x, out)]),
             lambda: ctx.aif_cache_read([B.CacheRead(0, out, None)]), lambda: ctx.aif_cache_fork([0], [1]), lambda: ctx.aif_cache_copy([0], [1]),
             lambda: ctx.aif_cache_trim([0], 0, 1), lambda: ctx.aif_cache_compact())
    refused = []
    with torch.cuda.graph(g):
        for f in calls:
            try:
                f()
            except B.AifError as e:
                refused.append(e.status)
        y += 1
    assert refused == [B.AIF_EINVAL] * len(calls)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.all(y == 3.0) and ctx.aif_cache_len(1) == 0
    ctx.aif_cache_attend([B.CacheQuery(0, x, out)])
    torch.cuda.synchronize()
    assert torch.all(out == 1.0)


def test_on_a_stream_of_its_own(torch):
    _say("another stream, many calls in a row without waiting")
    rng = np.random.default_rng(12)
    ctx = make(torch, "bf16", 2, 1, 64, 32, pages=64)
    k, v = rows(rng, 120, 1, 64, "bf16"), rows(rng, 120, 1, 64, "bf16")
    dk, dv = dev(torch, k, "bf16"), dev(torch, v, "bf16")
    q = wl.round_storage(rng.standard_normal((30, 2, 64)).astype(np.float32), "bf16")
    dq = dev(torch, q, "bf16")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    outs = []
    with torch.cuda.stream(side):
        for t in range(0, 120, 4):                      # rows come four at a time, and are asked for at once
            ctx.aif_cache_append([B.CacheAppend(0, dk[t:t + 4], dv[t:t + 4])])
            out = torch.empty_like(dq)
            ctx.aif_cache_attend([B.CacheQuery(0, dq, out)])
            outs.append(out)
        ctx.aif_cache_free([0])
        ctx.aif_cache_append([B.CacheAppend(0, dv, dk)])
    side.synchronize()
    for i, t in enumerate(range(0, 120, 4)):
        compare("bf16", host(outs[i]), None, q, k[:t + 4], v[:t + 4], 0.125, what=f"after {t + 4} rows")


def test_from_the_user_network_through_the_cache_to_the_scores(torch):
    """Sec. 3.1 with the cache between its phases: what the asynchronous network leaves is held in 4 bits, extended by a branch, and
    scored; the scores are those of the same values given densely, bit for bit, and the cache's attention is the target attention's."""
    import oracle
    from paper_2511_12934_amd import runner as R
    _say("user network -> cache -> fork, append -> read -> score; attend")
    cfg = wl.CONFIGS["A3"].scaled(n_items=3000, seq_len=150, n_users=2, n_cand=700)
    ucfg = wl.USER_CONFIGS["U3"].scaled(n_users=2)
    umodel = wl.make_user_net_model(ucfg)
    users = wl.make_raw_users(ucfg, 2)
    uctx = R.make_user_context(ucfg, umodel, max_users=2, max_seq_len=max(u.seq.shape[0] for u in users))
    raw = [R.upload_raw_user(ucfg, u) for u in users]
    uctx.aif_user_precompute([r.req for r in raw])
    d = ucfg.d
    ctx = make(torch, "bf16", 1, 1, d, pages=64, queries=1000)
    seqs = [r.seq_out[:u.seq.shape[0]].reshape(-1, 1, d) for r, u in zip(raw, users)]
    ctx.aif_cache_append([B.CacheAppend(i, s, s) for i, s in enumerate(seqs)])
    ctx.aif_cache_fork([0, 1], [2, 3])
    new = dev(torch, rows(np.random.default_rng(2), 10, 1, d, "bf16", 0.1), "bf16")
    ctx.aif_cache_append([B.CacheAppend(2, new, new), B.CacheAppend(3, new[:3], new[:3])])
    torch.cuda.synchronize()
    for i in (0, 1):
        n_new = (10, 3)[i]
        want = ref.hold(np.concatenate([host(seqs[i]), host(new[:n_new])]))
        n = len(want)
        k, v = (torch.empty((n, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ctx.aif_cache_read([B.CacheRead(2 + i, k, v)])
        torch.cuda.synchronize()
        assert np.array_equal(host(k), want.reshape(n, d)) and np.array_equal(host(v), want.reshape(n, d))
        gk, _ = read(torch, ctx, "bf16", i, 1, d)
        assert np.array_equal(gk, ref.hold(host(seqs[i])))               # the branch left its parent alone
        # the candidates' attention block of the scoring path over the unpacked rows, and the cache's own
        rng = np.random.default_rng(20 + i)
        model = wl.make_model(cfg)
        table = wl.make_table_host(cfg, rng, n_items=cfg.n_items)
        user = wl.make_user(cfg, rng)
        user.seq_keys = user.seq_vals = host(k)
        ids = wl.IdSampler(cfg, cfg.n_items).sample(rng, cfg.n_cand)
        dm, table_dev = R.DeviceModel(cfg, model), R.to_device(table, cfg.dtype)
        sctx = R.make_context(cfg, dm, table_dev, max_users=1, max_candidates=cfg.n_cand, max_seq_len=n)
        dr = R.upload_request(cfg, user, ids)
        sctx.aif_score_batch([dr.req])
        torch.cuda.synchronize()
        by_hand = host(dr.logits)
        dr.req.seq_keys, dr.req.seq_vals = k, v
        sctx.aif_score_batch([dr.req])
        torch.cuda.synchronize()
        assert np.array_equal(host(dr.logits), by_hand)
        z = oracle.score(table=table, ids=ids, user_vec=user.user_vec, seq_keys=user.seq_keys, seq_vals=user.seq_vals, dims=model.dims,
                         weights=model.weights, biases=model.biases, w_q=model.w_q, n_heads=cfg.n_heads, cross_mode=cfg.cross_mode,
                         cross_vecs=user.cross_vecs).logits
        assert np.abs(by_hand - z).max() <= 2e-2
        check_attend(torch, ctx, "bf16", 2 + i, np.concatenate([host(seqs[i]), host(new[:n_new])]), np.concatenate([host(seqs[i]), host(new[:n_new])]),
                     table[ids][:, None, :d], scale=d ** -0.5, what="candidates over the branch")
