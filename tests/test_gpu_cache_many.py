"""The user cache's attention where rows are many (candidates): large tiles, padded heads, mixed calls; against the 64-bit reference."""
import numpy as np
import pytest

from paper_2511_12934_amd import binding as B
from paper_2511_12934_amd import workloads as wl

from test_gpu_cache import _say, check_attend, compare, dev, fill, host, make, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


@pytest.mark.parametrize("dtype,heads,kv,d", [("bf16", 8, 8, 16), ("bf16", 8, 8, 64), ("bf16", 16, 4, 128), ("bf16", 8, 8, 40), ("bf16", 12, 6, 96),
                                              ("bf16", 4, 4, 160), ("f32", 8, 8, 16), ("f32", 4, 4, 64), ("f32", 2, 2, 192)])
@pytest.mark.parametrize("window", (0, 60))
def test_candidates_of_several_users(torch, dtype, heads, kv, d, window):
    """Enough (row tile, kv head) pairs for the widest tiles; sampled rows are compared."""
    _say(f"many rows {dtype} heads={heads}/{kv} d={d} window={window}")
    rng = np.random.default_rng(d + window)
    n_users, n_q = 10, 2000
    ctx = make(torch, dtype, heads, kv, d, 64, pages=120, seqs=n_users, requests=n_users, queries=n_q)
    asks, keep = [], []
    for u in range(n_users):
        n = (1, 33, 64, 100, 200, 257, 300, 31, 129, 500)[u]
        k, v = rows(rng, n, kv, d, dtype), rows(rng, n, kv, d, dtype)
        fill(torch, ctx, dtype, u, k, v)
        q = wl.round_storage(rng.standard_normal((n_q, heads, d)).astype(np.float32), dtype)
        pos = np.sort(rng.integers(-1, n + 3, n_q)) if window else None
        dq = dev(torch, q, dtype)
        out, lse = torch.full_like(dq, float("nan")), torch.full((n_q, heads), float("nan"), device="cuda")
        asks.append(B.CacheQuery(u, dq, out, lse=lse, window=window, sinks=3, positions=None if pos is None else torch.from_numpy(pos.astype(np.int32)).cuda()))
        keep.append((k, v, q, pos, out, lse))
    ctx.aif_cache_attend(asks)
    torch.cuda.synchronize()
    at = np.unique(np.concatenate([rng.integers(0, n_q, 25), [0, 1, n_q - 1]]))
    for u, (k, v, q, pos, out, lse) in enumerate(keep):
        compare(dtype, host(out)[at], host(lse)[at], q[at], k, v, d ** -0.5, positions=None if pos is None else pos[at], sinks=3, window=window, what=f"user {u}")


@pytest.mark.parametrize("dtype,heads,kv,d", [("bf16", 2, 2, 40), ("f32", 2, 2, 20), ("bf16", 4, 2, 16), ("f32", 2, 1, 100), ("bf16", 2, 1, 224)])
@pytest.mark.parametrize("n_q", (1, 300))
def test_nan_in_the_last_block_of_a_padded_head(torch, dtype, heads, kv, d, n_q):
    _say(f"NaN beside padding {dtype} d={d} n_q={n_q}")
    rng = np.random.default_rng(d)
    n = 100
    ctx = make(torch, dtype, heads, kv, d)
    k, v = rows(rng, n, kv, d, dtype), rows(rng, n, kv, d, dtype)
    v[40, 0, d - 1] = np.inf
    v[70, kv - 1, 0] = np.nan
    fill(torch, ctx, dtype, 0, k, v)
    q = wl.round_storage(rng.standard_normal((n_q, heads, d)).astype(np.float32), dtype)
    pos = rng.integers(0, n, n_q)
    pos[-1] = 39
    check_attend(torch, ctx, dtype, 0, k, v, q, scale=d ** -0.5, positions=pos, what="all before")
    check_attend(torch, ctx, dtype, 0, k, v, q, scale=d ** -0.5, positions=pos, window=5, sinks=2, what="window")


def test_few_and_many_rows_in_one_call_over_long_histories(torch):
    """Both kernels in one call, split keys in both, entries without queries between them."""
    _say("mixed call, split keys")
    rng = np.random.default_rng(4)
    heads, kv, d = 4, 2, 64
    ctx = make(torch, "bf16", heads, kv, d, 128, pages=200, seqs=4, longest=9000, requests=40, queries=400)
    data = []
    for s, n in enumerate((9000, 4100, 37, 0)):
        k, v = rows(rng, n, kv, d, "bf16"), rows(rng, n, kv, d, "bf16")
        fill(torch, ctx, "bf16", s, k, v)
        data.append((k, v))
    for n_req in (8, 40):
        asks, keep = [], []
        for r in range(n_req):
            s, n_q = r % 4, (1, 0, 400, 33, 150, 17)[r % 6]
            q = wl.round_storage(rng.standard_normal((n_q, heads, d)).astype(np.float32), "bf16")
            dq = dev(torch, q, "bf16")
            out, lse = torch.full_like(dq, float("nan")), torch.full((n_q, heads), float("nan"), device="cuda")
            asks.append(B.CacheQuery(s, dq, out, lse=lse))
            keep.append((s, q, out, lse))
        ctx.aif_cache_attend(asks)
        torch.cuda.synchronize()
        for s, q, out, lse in keep:
            if len(q):
                at = np.unique(rng.integers(0, len(q), 6))
                compare("bf16", host(out)[at], host(lse)[at], q[at], *data[s], d ** -0.5, what=f"sequence {s}, {len(q)} queries")


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f32", 40), ("bf16", 256)])
@pytest.mark.parametrize("n_q", (1, 200))
def test_dropped_pages_inside_what_is_seen(torch, dtype, d, n_q):
    _say(f"dropped pages {dtype} d={d} n_q={n_q}")
    rng = np.random.default_rng(9)
    n, kv = 700, 1
    ctx = make(torch, dtype, 2, kv, d, 32, pages=30)
    k, v = rows(rng, n, kv, d, dtype), rows(rng, n, kv, d, dtype)
    fill(torch, ctx, dtype, 0, k, v)
    ctx.aif_cache_trim([0], sinks=40, window=300)           # pages 2..11
    gone = ((64, 384),)
    other = rows(rng, 320, kv, d, dtype)
    fill(torch, ctx, dtype, 1, other, other)                # takes the pages that were given back
    q = wl.round_storage(rng.standard_normal((n_q, 2, d)).astype(np.float32), dtype)
    check_attend(torch, ctx, dtype, 0, k, v, q, scale=d ** -0.5, dropped=gone, what="all")
    pos = rng.integers(0, n, n_q)
    pos[0] = 200
    check_attend(torch, ctx, dtype, 0, k, v, q, scale=d ** -0.5, positions=pos, dropped=gone, what="positions")
    check_attend(torch, ctx, dtype, 0, k, v, q, scale=d ** -0.5, positions=pos, window=50, dropped=gone, what="window alone")
    check_attend(torch, ctx, dtype, 0, k, v, q, scale=d ** -0.5, sinks=40, window=300, dropped=gone, what="what trim keeps")
