"""The user cache where sizes and routes are the rare ones: pages beyond 4 GB, the copied descriptors, calls that are too large, pools that change."""
import gc
import weakref

import numpy as np
import pytest

import cache_reference as ref
from paper_2511_12934_amd import binding as B
from paper_2511_12934_amd import workloads as wl

from test_gpu_cache import _say, check_attend, compare, dev, fill, make, read, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def test_pages_beyond_four_gigabytes(torch):
    _say("pages beyond 4 GB")
    rng = np.random.default_rng(1)
    shape = dict(dtype=B.AIF_BF16, n_heads=8, n_kv_heads=8, d_head=256, page_len=1024)
    page = B.cache_page_bytes(**shape)
    each = 64                                                   # pages of one of the long sequences
    n = -(-(1 << 32) // (each * page)) + 1                      # so many of them lie before the one that is looked at
    pool = torch.empty(((n * each + 2) * page,), dtype=torch.uint8, device="cuda")
    ctx = B.CacheContext(pool=pool, max_seqs=n + 2, max_len=each * 1024, max_requests=4, max_queries=70, **shape)
    ones = torch.ones((each * 1024, 8, 256), dtype=torch.bfloat16, device="cuda")
    ctx.aif_cache_append([B.CacheAppend(0, ones, ones)])
    ctx.aif_cache_copy([0] * (n - 1), list(range(1, n)))
    del ones
    k, v = rows(rng, 300, 8, 256, "bf16"), rows(rng, 300, 8, 256, "bf16")
    fill(torch, ctx, "bf16", n, k, v)
    assert ctx.aif_cache_free_pages() == 1
    gk, gv = read(torch, ctx, "bf16", n, 8, 256)
    assert np.array_equal(gk, ref.hold(k)) and np.array_equal(gv, ref.hold(v))
    q = wl.round_storage(rng.standard_normal((70, 8, 256)).astype(np.float32), "bf16")
    check_attend(torch, ctx, "bf16", n, k, v, q[:1], scale=1 / 16, what="one query")
    check_attend(torch, ctx, "bf16", n, k, v, q, scale=1 / 16, what="70 queries")
    ctx.aif_cache_copy([n], [n + 1])
    ctx.aif_cache_free(list(range(n)))
    assert ctx.aif_cache_compact() == 2
    check_attend(torch, ctx, "bf16", n + 1, k, v, q[:3], scale=1 / 16, what="moved")
    assert np.array_equal(read(torch, ctx, "bf16", n, 8, 256)[0], ref.hold(k))


def test_descriptors_that_are_copied_to_the_device(torch, monkeypatch):
    """The route of a host whose pinned memory is not mapped, with more descriptors than a launch's arguments hold."""
    _say("descriptors by copy")
    results = []
    for copied in (False, True):
        if copied:
            monkeypatch.setenv("AIF_STAGING_COPY", "1")
        rng = np.random.default_rng(2)
        n = 150
        ctx = make(torch, "bf16", 2, 1, 32, 32, pages=4 * n, seqs=2 * n, longest=100, requests=n, queries=4)
        data = [rows(rng, int(m), 1, 32, "bf16") for m in rng.integers(0, 100, n)]
        ctx.aif_cache_append([B.CacheAppend(u, dev(torch, x, "bf16"), dev(torch, x, "bf16")) for u, x in enumerate(data)])
        some = list(range(0, n, 2))
        ctx.aif_cache_fork(some, [n + u for u in some])
        ctx.aif_cache_free(some)
        q = dev(torch, rng.standard_normal((n, 2, 2, 32)), "bf16")
        out = torch.full_like(q, float("nan"))
        ctx.aif_cache_attend([B.CacheQuery(u + (n if u % 2 == 0 else 0), q[u], out[u]) for u in range(n)])
        back = [torch.zeros((len(x), 1, 32), dtype=torch.bfloat16, device="cuda") for x in data]
        ctx.aif_cache_read([B.CacheRead(u + (n if u % 2 == 0 else 0), b, None) for u, b in enumerate(back)])
        torch.cuda.synchronize()
        for b, x in zip(back, data):
            assert np.array_equal(b.float().cpu().numpy(), ref.hold(x))
        results.append(out.float().cpu().numpy())
    assert np.array_equal(results[0], results[1])


def test_calls_of_more_rows_than_their_numbers_reach_are_refused(torch):
    _say("too many rows")
    ctx = make(torch, "bf16", 4, 1, 64, requests=4, queries=2 ** 31 - 1)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    for n_q in (2 ** 29, 2 ** 30, 2 ** 31 - 1):
        r = B.pack_cache_queries([B.CacheQuery(0, q, torch.empty_like(q))])
        r[0].n_q = n_q
        assert ctx._lib.aif_cache_attend(ctx._h, r, 1, None) == B.AIF_ERANGE
        assert "too many" in ctx._lib.aif_cache_last_error(ctx._h).decode()


def test_a_pool_that_was_left_is_not_kept(torch):
    _say("pools that change")
    rng = np.random.default_rng(3)
    ctx = make(torch, "f32", 1, 1, 32, 32, pages=40, seqs=2, longest=600)
    k = rows(rng, 600, 1, 32, "f32")
    fill(torch, ctx, "f32", 0, k, k)
    first = weakref.ref(ctx._keep[0])
    assert ctx.aif_cache_compact() == 19
    pool = torch.empty((19 * B.cache_page_bytes(dtype=B.AIF_F32, n_heads=1, n_kv_heads=1, d_head=32, page_len=32),), dtype=torch.uint8, device="cuda")
    pool.copy_(ctx._keep[0][:pool.numel()])
    ctx.aif_cache_swap_pool(pool)
    gc.collect()
    assert first() is None
    q = wl.round_storage(rng.standard_normal((5, 1, 32)).astype(np.float32), "f32")
    check_attend(torch, ctx, "f32", 0, k, k, q, scale=32 ** -0.5, what="the new pool")


@pytest.mark.parametrize("n,n_q,longest", [(40, 1, 3000), (139, 1, 3000), (140, 1, 400), (100, 70, 200), (100, 300, 200), (300, 2, 100)])
@pytest.mark.parametrize("window", (0, 90))
def test_entries_alike_and_not_give_the_same_bits(torch, n, n_q, longest, window):
    """Queries and outputs of a batch in one tensor each, and the same with one entry's output elsewhere."""
    _say(f"{n} entries alike, {n_q} queries, window {window}")
    rng = np.random.default_rng(n + n_q)
    heads, kv, d = 4, 2, 64
    ctx = make(torch, "bf16", heads, kv, d, 64, pages=n * (longest // 64 + 1), seqs=n, longest=longest, requests=n, queries=n_q)
    source = dev(torch, rows(rng, longest, kv, d, "bf16"), "bf16")
    lens = rng.integers(0, longest + 1, n)
    lens[n - 1] = longest
    ctx.aif_cache_append([B.CacheAppend(u, source[longest - m:], source[longest - m:]) for u, m in enumerate(lens)])
    q_host = wl.round_storage(rng.standard_normal((n, n_q, heads, d)).astype(np.float32), "bf16")
    q = dev(torch, q_host, "bf16")
    where = rng.integers(-1, longest, (n, n_q)).astype(np.int32)
    at = torch.from_numpy(where).cuda()
    got = []
    for apart in (False, True):
        out, lse = torch.full_like(q, float("nan")), torch.full((n, n_q, heads), float("nan"), device="cuda")
        outs = [out[u] for u in range(n)]
        if apart:
            outs[n // 2] = torch.full_like(q[0], float("nan"))
        ctx.aif_cache_attend([B.CacheQuery(u, q[u], outs[u], lse=lse[u], positions=at[u] if window else None, window=window, sinks=3) for u in range(n)])
        torch.cuda.synchronize()
        got.append((torch.stack(outs).float().cpu().numpy(), lse.cpu().numpy()))
    assert np.array_equal(got[0][0], got[1][0]) and np.array_equal(got[0][1], got[1][1])
    held = source.float().cpu().numpy()
    some = slice(0, 4)
    for u in (0, n // 2, n - 1):
        k = held[longest - lens[u]:]
        compare("bf16", got[0][0][u][some], got[0][1][u][some], q_host[u][some], k, k, d ** -0.5, positions=where[u][some] if window else None, sinks=3, window=window, what=f"entry {u}")


@pytest.mark.parametrize("dtype,kv,d,pl", [("bf16", 2, 64, 32), ("f32", 1, 40, 96)])
def test_copies_into_a_pool_of_scattered_pages(torch, dtype, kv, d, pl):
    """More runs of pages than a launch's arguments hold, dropped pages among them, rows read from the middle of pages."""
    _say(f"scattered copies {dtype} page={pl}")
    rng = np.random.default_rng(pl)
    n_pages = 220
    longest = n_pages * pl
    ctx = make(torch, dtype, kv, kv, d, pl, pages=3 * n_pages, seqs=5, longest=longest, requests=2)
    k, v = rows(rng, longest - 5, kv, d, dtype), rows(rng, longest - 5, kv, d, dtype)
    dk, dv = dev(torch, k, dtype), dev(torch, v, dtype)
    for lo in range(0, longest - 5, pl):
        ctx.aif_cache_append([B.CacheAppend(u, dk[lo:lo + pl], dv[lo:lo + pl]) for u in (0, 1)])
    ctx.aif_cache_fork([0], [2])
    ctx.aif_cache_trim([2], sinks=10, window=longest - 9 * pl)
    ctx.aif_cache_free([1])
    ctx.aif_cache_copy([0, 2], [3, 4])
    hk, hv = ref.hold(k), ref.hold(v)
    for first, n in ((0, longest - 5), (pl - 1, 2), (7, 1), (5 * pl + 3, 3 * pl), (longest - 6, 1), (longest - 5, 0)):
        gk, gv = read(torch, ctx, dtype, 3, kv, d, first=first, n=n)
        assert np.array_equal(gk, hk[first:first + n]) and np.array_equal(gv, hv[first:first + n]), (first, n)
    gk, _ = read(torch, ctx, dtype, 4, kv, d, first=10 * pl, n=4 * pl)
    assert np.array_equal(gk, hk[10 * pl:14 * pl])
    with pytest.raises(B.AifError, match="dropped"):
        read(torch, ctx, dtype, 4, kv, d, first=2 * pl, n=1)
    q = wl.round_storage(rng.standard_normal((2, kv, d)).astype(np.float32), dtype)
    gone = ((pl, (longest - 5 - (longest - 9 * pl)) // pl * pl),)
    check_attend(torch, ctx, dtype, 4, k, v, q, scale=d ** -0.5, dropped=gone, what="a copy with dropped pages")


def test_a_history_onto_scattered_pages(torch):
    """Rows appended to more runs of pages than a launch's arguments hold, the first of them a shared page."""
    _say("an append onto scattered pages")
    rng = np.random.default_rng(8)
    pl, d, n_pages = 32, 32, 300
    ctx = make(torch, "bf16", 1, 1, d, pl, pages=n_pages, seqs=n_pages + 2, longest=n_pages * pl, requests=n_pages)
    some = rows(rng, n_pages * pl, 1, d, "bf16")
    t = dev(torch, some, "bf16")
    ctx.aif_cache_append([B.CacheAppend(u, t[u:u + 20], t[u:u + 20]) for u in range(n_pages)])
    ctx.aif_cache_free(list(range(0, n_pages, 2)))
    ctx.aif_cache_fork([1, 1], [n_pages, n_pages + 1])
    more = 140 * pl
    ctx.aif_cache_append([B.CacheAppend(n_pages, t[:more], t[:more]), B.CacheAppend(n_pages + 1, t[5:9], t[5:9])])
    want = np.concatenate([some[1:21], some[:more]])
    assert np.array_equal(read(torch, ctx, "bf16", n_pages, 1, d)[0], ref.hold(want))
    assert np.array_equal(read(torch, ctx, "bf16", n_pages + 1, 1, d)[1], ref.hold(np.concatenate([some[1:21], some[5:9]])))
    for u in (1, 3, 151, n_pages - 1):
        assert np.array_equal(read(torch, ctx, "bf16", u, 1, d)[0], ref.hold(some[u:u + 20])), u


@pytest.mark.parametrize("dtype,n", [("bf16", 70), ("f32", 700)])
def test_many_unlike_entries_in_one_call(torch, dtype, n):
    """More entries than a wave has lanes: appends, queries and reads of unlike lengths, some of none."""
    _say(f"{n} unlike entries {dtype}")
    rng = np.random.default_rng(n)
    kv, heads, d, pl = 2, 4, 40, 64
    ctx = make(torch, dtype, heads, kv, d, pl, pages=6 * n, seqs=n, longest=300, requests=n, queries=90)
    lens, n_qs = rng.integers(0, 300, n), rng.integers(0, 3, n) * rng.integers(0, 45, n)
    lens[::7], n_qs[5::9] = 0, 1
    k, v = rows(rng, 400, kv, d, dtype), rows(rng, 400, kv, d, dtype)
    dk, dv = dev(torch, k, dtype), dev(torch, v, dtype)
    cuts = np.minimum(lens, rng.integers(0, 300, n))
    ctx.aif_cache_append([B.CacheAppend(u, dk[u % 90:u % 90 + cuts[u]], dv[u % 90:u % 90 + cuts[u]]) for u in range(n)])
    ctx.aif_cache_append([B.CacheAppend(u, dk[u % 90 + cuts[u]:u % 90 + lens[u]], dv[u % 90 + cuts[u]:u % 90 + lens[u]]) for u in rng.permutation(n)])
    order = rng.permutation(n)
    q_host = wl.round_storage(rng.standard_normal((90, heads, d)).astype(np.float32), dtype)
    q = dev(torch, q_host, dtype)
    outs = {u: torch.full_like(q[:n_qs[u]], float("nan")) for u in order}
    lse = {u: torch.full((int(n_qs[u]), heads), float("nan"), device="cuda") for u in order}
    ctx.aif_cache_attend([B.CacheQuery(int(u), q[:n_qs[u]], outs[u], lse=lse[u]) for u in order])
    back = [torch.zeros((int(m), kv, d), device="cuda").to(dk.dtype) for m in lens]
    ctx.aif_cache_read([B.CacheRead(int(u), None, back[u]) for u in order])
    torch.cuda.synchronize()
    for u in range(n):
        assert np.array_equal(back[u].float().cpu().numpy(), ref.hold(v[u % 90:u % 90 + lens[u]])), u
    for u in [int(x) for x in order if n_qs[x]][:25]:
        at = slice(u % 90, u % 90 + int(lens[u]))
        compare(dtype, outs[u].float().cpu().numpy(), lse[u].cpu().numpy(), q_host[:n_qs[u]], k[at], v[at], d ** -0.5, what=f"entry {u}")
