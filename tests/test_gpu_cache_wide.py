"""The kernels that serve calls of very many rows: entries of 65 rows and more beside one that fills the device, against the 64-bit reference."""
import numpy as np
import pytest

from paper_2511_12934_amd import binding as B
from paper_2511_12934_amd import workloads as wl

from test_gpu_cache import _say, compare, dev, fill, host, make, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


WIDTHS = [("bf16", 2, 2, 16), ("bf16", 4, 2, 64), ("bf16", 2, 1, 40), ("f32", 2, 2, 32), ("f32", 2, 1, 64), ("bf16", 3, 3, 96), ("bf16", 4, 2, 128), ("bf16", 2, 2, 160),
          ("bf16", 1, 1, 192), ("bf16", 2, 1, 224), ("bf16", 2, 2, 256), ("f32", 2, 2, 96), ("f32", 4, 2, 128), ("f32", 1, 1, 160), ("f32", 1, 1, 192), ("f32", 2, 1, 224),
          ("f32", 1, 1, 256)]


class Call:
    """Entries of one attend call, each with what it has to give."""

    def __init__(self, torch, ctx, dtype, heads, d, rng):
        self.torch, self.ctx, self.dtype, self.heads, self.d, self.rng = torch, ctx, dtype, heads, d, rng
        self.asks, self.checks = [], []

    def add(self, seq, data, n_q, *, positions=None, sinks=0, window=0, gap=0, times=1.0, sample=None, what=""):
        t, width = self.torch, self.heads * self.d
        q = wl.round_storage((times * self.rng.standard_normal((n_q, self.heads, self.d))).astype(np.float32), self.dtype)
        dq = dev(t, q, self.dtype)
        if gap:
            room = [t.full((n_q, width + gap), 5.0, device="cuda", dtype=dq.dtype) for _ in range(2)]
            room[0][:, :width] = dq.reshape(n_q, width)
            dq, out = (x[:, :width].unflatten(1, (self.heads, self.d)) for x in room)
        else:
            room, out = None, t.full_like(dq, float("nan"))
        lse = t.full((n_q, self.heads), float("nan"), device="cuda")
        at = None if positions is None else t.from_numpy(np.asarray(positions, np.int32)).cuda()
        self.asks.append(B.CacheQuery(seq, dq, out, lse=lse, positions=at, sinks=sinks, window=window))
        pick = np.arange(n_q) if sample is None else np.unique(np.concatenate([self.rng.integers(0, n_q, sample), [0, n_q - 1]]))

        def check():
            o, l = host(out)[pick], host(lse)[pick]
            compare(self.dtype, o, l, q[pick], *data, self.d ** -0.5, None if positions is None else np.asarray(positions)[pick], sinks, window, what=what)
            if gap:
                assert (room[1][:, width:] == 5).all(), f"{what}: wrote beside its rows"
        self.checks.append(check)

    def run(self):
        self.ctx.aif_cache_attend(self.asks)
        self.torch.cuda.synchronize()
        for check in self.checks:
            check()


@pytest.mark.parametrize("dtype,heads,kv,d,whole", [(*w, 20000) for w in WIDTHS] + [(*w, 140000) for w in WIDTHS if w[0] == "bf16" and w[3] <= 128])
def test_entries_beside_one_that_fills_the_device(torch, dtype, heads, kv, d, whole):
    """`whole`: rows of the entry that fills it, for row tiles of 128 and, where there are any, of 256."""
    _say(f"beside {whole} rows: {dtype} heads={heads}/{kv} d={d}")
    rng = np.random.default_rng(d + whole)
    group = heads // kv
    ctx = make(torch, dtype, heads, kv, d, 64, pages=130, seqs=6, longest=3600, requests=16, queries=150000)
    data = []
    for s, n in enumerate((500, 33, 1, 0, 3500, 300)):
        k, v = rows(rng, n, kv, d, dtype), rows(rng, n, kv, d, dtype)
        if s == 5:
            v[100, 0, d - 1], k[200, kv - 1, 0] = np.inf, np.nan
        fill(torch, ctx, dtype, s, k, v)
        data.append((k, v))
    some = -(-65 // group)              # 65 rows and a few
    for windows in (False, True):
        call = Call(torch, ctx, dtype, heads, d, rng)
        call.add(0, data[0], some, what="few")
        call.add(1, data[1], -(-whole // heads), sample=20, what="the large one")
        call.add(4, data[4], 2 * some + 3, sample=40, what="long")
        call.add(2, data[2], some, what="one key")
        call.add(3, data[3], some, what="no keys")
        call.add(0, data[0], 2, what="two queries")
        call.add(0, data[0], 130, gap=24, times=30.0, sample=40, what="rows apart, large scores")
        order = rng.integers(0, 500, 140)
        order[[0, 5, 131]] = -7, 10 ** 9, -1
        call.add(0, data[0], 140, positions=order, sample=60, what="positions")
        early = np.sort(rng.integers(0, 300, 90))
        early[:9] = 99
        call.add(5, data[5], 90, positions=early, what="not finite")
        if windows:
            call.add(0, data[0], 140, positions=order, window=60, sinks=3, sample=60, what="window")
            call.add(5, data[5], 90, positions=early, window=40, sinks=1, what="not finite, window")
            call.add(4, data[4], 100, positions=np.full(100, -3), window=5, what="all rows see nothing")
            call.add(4, data[4], 100, window=300, sinks=2, sample=30, what="window at the end")
        call.run()


@pytest.mark.parametrize("dtype,kv,d", [("bf16", 1, 64), ("bf16", 2, 128), ("f32", 1, 64), ("bf16", 1, 256)])
@pytest.mark.parametrize("n_users,n_q", [(130, 8), (130, 64), (257, 130), (3, 5500)])
def test_short_and_long_sequences_at_every_way_to_cut_the_work(torch, dtype, kv, d, n_users, n_q):
    """Sequences shared out over blocks and not, row tiles fewer and more than the device holds."""
    _say(f"cuts {dtype} kv={kv} d={d} {n_users} x {n_q}")
    rng = np.random.default_rng(n_users + n_q)
    ctx = make(torch, dtype, kv, kv, d, 64, pages=3 * n_users + 170, seqs=n_users, longest=9000, requests=n_users, queries=n_q)
    call = Call(torch, ctx, dtype, kv, d, rng)
    for u in range(n_users):
        n = 9000 if u == 1 else int(rng.integers(0, 180))
        data = rows(rng, n, kv, d, dtype), rows(rng, n, kv, d, dtype)
        fill(torch, ctx, dtype, u, *data)
        call.add(u, data, n_q, sample=3, what=f"user {u}")
    call.run()
