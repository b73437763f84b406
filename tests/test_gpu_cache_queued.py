"""The user cache's calls one after the other without waiting between them, against the 64-bit reference."""
import numpy as np
import pytest

import cache_reference as ref
from paper_2511_12934_amd import binding as B

from test_gpu_cache import _say, compare, dev, make, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


@pytest.mark.parametrize("copied", (False, True))
def test_descriptors_of_queued_calls_are_left_alone(torch, monkeypatch, copied):
    """Calls one after the other without waiting, whose descriptors fill both halves of the memory that they wait in twice and more."""
    _say(f"queued calls, descriptors {'copied' if copied else 'mapped'}")
    if copied:
        monkeypatch.setenv("AIF_STAGING_COPY", "1")
    rng = np.random.default_rng(13)
    n, d, longest = 600, 32, 40
    ctx = make(torch, "bf16", 1, 1, d, 32, pages=6 * n, seqs=3 * n, longest=longest, requests=n, queries=4)
    data = [rows(rng, int(m), 1, d, "bf16") for m in rng.integers(1, longest - 2, n)]
    whole = dev(torch, np.concatenate(data), "bf16")
    cut = np.concatenate([[0], np.cumsum([len(x) for x in data])])
    ctx.aif_cache_append([B.CacheAppend(u, whole[cut[u]:cut[u + 1]], whole[cut[u]:cut[u + 1]]) for u in range(n)])
    ctx.aif_cache_copy(list(range(n)), list(range(n, 2 * n)))
    q = dev(torch, rng.standard_normal((n, 4, 1, d)), "bf16")
    once = []
    for of in (0, n):                   # what a call of its own gives: sequences u and u + n hold the same
        out = torch.full_like(q, float("nan"))
        for lo in range(0, n, 30):
            ctx.aif_cache_attend([B.CacheQuery(of + u, q[u, :1 + u % 4], out[u, :1 + u % 4]) for u in range(lo, lo + 30)])
            torch.cuda.synchronize()
        once.append(out)
    assert torch.equal(once[0].nan_to_num(7.0), once[1].nan_to_num(7.0))
    torch.cuda.synchronize()
    results, reads, orders = [], [], []
    for turn in range(36):              # a call's descriptors take about 62 KB (queries), 29 KB (reads), 10 KB (branches): 3.6 MB, of halves of 1 MB
        order = rng.permutation(n)
        out = torch.full_like(q, float("nan"))
        of = n * (turn % 3)
        if of == 2 * n:
            ctx.aif_cache_free(list(range(2 * n, 3 * n)))
            ctx.aif_cache_fork(order, 2 * n + order)
        ctx.aif_cache_attend([B.CacheQuery(of + int(u), q[u, :1 + u % 4], out[u, :1 + u % 4]) for u in order])
        back = torch.zeros_like(whole)
        ctx.aif_cache_read([B.CacheRead(of + int(u), back[cut[u]:cut[u + 1]], None) for u in order])
        results.append(out), reads.append(back), orders.append(order)
    torch.cuda.synchronize()
    held = ref.hold(np.concatenate(data))
    for turn, (out, back) in enumerate(zip(results, reads)):
        assert np.array_equal(back.float().cpu().numpy(), held), turn
        assert torch.equal(out.nan_to_num(7.0), once[0].nan_to_num(7.0)), turn
    for u in (0, 1, 2, 3, n - 1):
        compare("bf16", results[-1][u, :1 + u % 4].float().cpu().numpy(), None, q[u, :1 + u % 4].float().cpu().numpy(), data[u], data[u], d ** -0.5, what=f"entry {u}")
