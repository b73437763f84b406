"""The user cache with the narrowest heads there are, one row that lies in a wider tensor, and requests packed beforehand, against the 64-bit reference."""
import numpy as np
import pytest

import cache_reference as ref
from paper_2511_12934_amd import binding as B
from paper_2511_12934_amd import workloads as wl

from test_gpu_cache import _say, check_attend, compare, dev, fill, host, make, read, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


@pytest.mark.parametrize("dtype,heads,kv,d", [("bf16", 1, 1, 8), ("bf16", 6, 2, 24), ("f32", 1, 1, 4), ("f32", 4, 2, 12), ("f32", 3, 3, 36)])
@pytest.mark.parametrize("n,n_q", [(1, 1), (45, 3), (300, 40)])
def test_narrow_heads(torch, dtype, heads, kv, d, n, n_q):
    _say(f"narrow heads {dtype} {heads}/{kv} d={d} n={n} n_q={n_q}")
    rng = np.random.default_rng(d + n)
    ctx = make(torch, dtype, heads, kv, d, 32)
    k, v = rows(rng, n, kv, d, dtype), rows(rng, n, kv, d, dtype)
    fill(torch, ctx, dtype, 0, k, v, cuts=(n // 2,))
    gk, gv = read(torch, ctx, dtype, 0, kv, d)
    assert np.array_equal(gk, ref.hold(k)) and np.array_equal(gv, ref.hold(v))
    q = wl.round_storage(rng.standard_normal((n_q, heads, d)).astype(np.float32), dtype)
    check_attend(torch, ctx, dtype, 0, k, v, q, scale=d ** -0.5, what="whole")
    check_attend(torch, ctx, dtype, 0, k, v, q, scale=d ** -0.5, positions=rng.integers(-1, n + 2, n_q), window=7, sinks=2, what="window")


@pytest.mark.parametrize("dtype,d", [("bf16", 8), ("f32", 4), ("bf16", 24), ("f32", 12)])
def test_narrow_heads_of_many_candidates(torch, dtype, d):
    _say(f"narrow heads, many rows {dtype} d={d}")
    rng = np.random.default_rng(d)
    heads, n, n_q = 4, 200, 9000
    ctx = make(torch, dtype, heads, heads, d, 64, queries=n_q)
    k, v = rows(rng, n, heads, d, dtype), rows(rng, n, heads, d, dtype)
    fill(torch, ctx, dtype, 0, k, v)
    q = wl.round_storage(rng.standard_normal((n_q, heads, d)).astype(np.float32), dtype)
    dq = dev(torch, q, dtype)
    out, lse = torch.full_like(dq, float("nan")), torch.full((n_q, heads), float("nan"), device="cuda")
    ctx.aif_cache_attend([B.CacheQuery(0, dq, out, lse=lse)])
    torch.cuda.synchronize()
    at = np.unique(np.concatenate([rng.integers(0, n_q, 30), [0, n_q - 1]]))
    compare(dtype, host(out)[at], host(lse)[at], q[at], k, v, d ** -0.5, what="candidates")


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_one_row_of_wider_tensors(torch, dtype):
    """A single behaviour and a single query, as views of fused projections whose row lies close, and their neighbours left alone."""
    _say(f"one row of wider tensors {dtype}")
    rng = np.random.default_rng(4)
    heads, kv, d, n = 4, 2, 64, 40
    ctx = make(torch, dtype, heads, kv, d, 32)
    k, v = rows(rng, n, kv, d, dtype), rows(rng, n, kv, d, dtype)
    for t in range(n):
        kv_row = dev(torch, np.concatenate([k[t].reshape(1, -1), v[t].reshape(1, -1)], 1), dtype)      # [1, K | V]
        keys, vals = kv_row.chunk(2, -1)
        ctx.aif_cache_append([B.CacheAppend(0, keys, vals)])
    gk, gv = read(torch, ctx, dtype, 0, kv, d)
    assert np.array_equal(gk, ref.hold(k)) and np.array_equal(gv, ref.hold(v))
    q = wl.round_storage(rng.standard_normal((1, heads, d)).astype(np.float32), dtype)
    wide = torch.full((3, 3 * heads * d), 5.0, device="cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16)
    part = slice(heads * d, 2 * heads * d)
    wide[1, part] = dev(torch, q.reshape(-1), dtype)
    res = torch.full_like(wide, 3.0)
    ctx.aif_cache_attend([B.CacheQuery(0, wide[1:2, part], res[1:2, part])])
    torch.cuda.synchronize()
    compare(dtype, host(res[1:2, part]).reshape(1, heads, d), None, q, k, v, d ** -0.5, what="one query")
    res[1, part] = 3.0
    assert torch.all(res == 3.0)
    one = torch.full_like(wide, 3.0)
    ctx.aif_cache_read([B.CacheRead(0, one[2:, :kv * d], one[2:, 2 * kv * d:3 * kv * d], first=17)])
    assert np.array_equal(host(one[2, :kv * d]).reshape(kv, d), ref.hold(k)[17])
    one[2, :kv * d] = one[2, 2 * kv * d:3 * kv * d] = 3.0
    assert torch.all(one == 3.0)
    fused = torch.zeros((1, kv, 2 * d), device="cuda").to(wide.dtype)
    with pytest.raises(ValueError, match="contiguous"):
        ctx.aif_cache_append([B.CacheAppend(0, *fused.chunk(2, -1))])
    assert ctx.aif_cache_len(0) == n


def test_packed_requests_of_another_context_are_refused(torch):
    _say("packed requests of another context")
    a, b = make(torch, "bf16", 2, 1, 64), make(torch, "f32", 2, 1, 64)
    x = torch.ones((3, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    appends, asks = [B.CacheAppend(0, x, x)], [B.CacheQuery(0, q, torch.zeros_like(q))]
    packed = B.pack_cache_appends(appends), B.pack_cache_queries(asks)
    for _ in range(2):
        a.aif_cache_append(appends, packed=packed[0])
        a.aif_cache_attend(asks, packed=packed[1])
        with pytest.raises(ValueError, match="the context 64 torch.float32"):
            b.aif_cache_append(appends, packed=packed[0])
        with pytest.raises(ValueError, match="the context 128 torch.float32"):
            b.aif_cache_attend(asks, packed=packed[1])
    with pytest.raises(ValueError, match="on cpu"):
        a.aif_cache_append([B.CacheAppend(0, x.cpu(), x.cpu())])
    with pytest.raises(ValueError, match="pool"):
        B.CacheContext(pool=torch.zeros(1 << 16, dtype=torch.uint8), dtype=B.AIF_BF16, n_heads=1, n_kv_heads=1, d_head=64, page_len=32, max_seqs=1,
                       max_len=32, max_requests=1)
    torch.cuda.synchronize()
    assert torch.all(asks[0].out == 1.0) and a.aif_cache_len(0) == 6 and b.aif_cache_len(0) == 0
