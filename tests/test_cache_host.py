"""The whole host side of the user cache on a queue in the place of the device (cache_host.cpp): rows are the addresses that they were given by,
launches read their descriptors when their turn comes, and any HIP call can be made to fail."""
import ctypes as C
import os
import random
import subprocess

import pytest

from paper_2511_12934_amd import binding as B
from paper_2511_12934_amd import build

OUT_OF_MEMORY, LAUNCH_FAILURE = 2, 719      # hipError_t


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("cache_host") / "cache_host.so")
    subprocess.check_call([build.HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-g", "-std=c++17", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-I", build.CSRC,
                           os.path.join(os.path.dirname(__file__), "cache_host.cpp"), "-o", so])
    lib = C.CDLL(so)
    B._declare_cache(lib)
    lib.host_fail.argtypes = [C.c_longlong, C.c_int]
    lib.host_calls.restype = lib.host_waiting.restype = C.c_longlong
    lib.host_wrong.restype = C.c_char_p
    lib.host_result.argtypes = [C.c_int64, C.POINTER(C.c_int64), C.c_int]
    return lib


class Cache:
    """A context and what its sequences hold: lists of row numbers, None for a dropped row."""
    WIDTH = 32                                  # of a key row, one head

    def __init__(self, lib, *, seqs, longest, pages, requests, page_len=32, n_heads=1, mapped=True, queries=8):
        self.lib, self.pl, self.seqs, self.pages = lib, page_len, seqs, pages
        lib.host_reset(pages, page_len, int(mapped))
        cfg = B.aif_cache_config(B.AIF_BF16, n_heads, 1, self.WIDTH, 0.0, page_len, pages, seqs, longest, requests, queries)
        self.h = C.c_void_p()
        assert lib.aif_cache_init(C.byref(cfg), 64, C.byref(self.h)) == B.AIF_OK
        self.rows = [[] for _ in range(seqs)]
        self.next, self.next_out, self.wanted = 1 << 20, 1 << 44, []

    def close(self):
        self.lib.host_run()
        self.lib.aif_cache_destroy(self.h)

    def out(self):
        self.next_out += 1 << 20
        return self.next_out

    def append(self, named):
        arr = (B.aif_cache_append_req * len(named))()
        for r, (s, n) in zip(arr, named):
            r.seq, r.n_rows, r.keys, r.vals = s, n, self.next, self.next + (1 << 40)
            new = [self.next + 2 * self.WIDTH * i for i in range(n)]
            self.next += 2 * self.WIDTH * max(n, 1)
            r.new = new
        st = self.lib.aif_cache_append(self.h, arr, len(named), None)
        if st == B.AIF_OK:
            for r in range(len(named)):
                self.rows[named[r][0]] = self.rows[named[r][0]] + [arr[r].keys + 2 * self.WIDTH * i for i in range(named[r][1])]
        return st

    def attend(self, asks, even=False):
        """[(sequence, queries)]; even: outputs that lie evenly."""
        arr = (B.aif_cache_attend_req * len(asks))()
        step = self.out()
        for i, (r, (s, n)) in enumerate(zip(arr, asks)):
            r.seq, r.n_q, r.q = s, n, 4096
            r.out = step + (i << 12) if even else step + (i << 12) + (i * i % 3 << 8)
        self.next_out += len(asks) << 12
        st = self.lib.aif_cache_attend(self.h, arr, len(asks), None)
        if st == B.AIF_OK:
            self.wanted += [(arr[i].out, [-1 if x is None else x for x in self.rows[s]]) for i, (s, n) in enumerate(asks) if n]
        return st

    def read(self, parts):
        """[(sequence, first, n)]"""
        arr = (B.aif_cache_read_req * len(parts))()
        for r, (s, first, n) in zip(arr, parts):
            r.seq, r.first, r.n_rows = s, first, n
            r.keys_out, r.vals_out = self.out(), self.out()
        st = self.lib.aif_cache_read(self.h, arr, len(parts), None)
        if st == B.AIF_OK:
            for r, (s, first, n) in zip(arr, parts):
                self.wanted.append((r.keys_out, self.rows[s][first:first + n]))
                self.wanted.append((r.vals_out, [x + (1 << 40) for x in self.rows[s][first:first + n]]))
        return st

    def branch(self, what, src, dst):
        st = getattr(self.lib, "aif_cache_" + what)(self.h, B.cache_ids(src), B.cache_ids(dst), len(src), None)
        if st == B.AIF_OK:
            for a, b in zip(src, dst):
                self.rows[b] = list(self.rows[a])
        return st

    def trim(self, seqs, sinks, window):
        st = self.lib.aif_cache_trim(self.h, B.cache_ids(seqs), len(seqs), sinks, window, None)
        if st == B.AIF_OK:
            for s in seqs:
                for p in range(-(-sinks // self.pl), max(0, len(self.rows[s]) - window) // self.pl):
                    self.rows[s][p * self.pl:(p + 1) * self.pl] = [None] * self.pl
        return st

    def free(self, seqs):
        assert self.lib.aif_cache_free(self.h, B.cache_ids(seqs), len(seqs)) == B.AIF_OK
        for s in seqs:
            self.rows[s] = []

    def compact(self):
        return self.lib.aif_cache_compact(self.h, None, None)

    def free_pages(self):
        return self.lib.aif_cache_free_pages(self.h)

    def check(self, whole=True):
        """Everything that was asked for, and, `whole`, what every sequence holds now."""
        if whole:
            for s, rows in enumerate(self.rows):
                assert self.lib.aif_cache_len(self.h, s) == len(rows)
                if rows:
                    assert self.attend([(s, 1)]) == B.AIF_OK
        self.lib.host_run()
        for at, want in self.wanted:
            got = (C.c_int64 * max(len(want), 1))()
            n = self.lib.host_result(at, got, len(want))
            assert n == len(want) and list(got)[:n] == want, hex(at)
        self.wanted = []
        assert self.lib.host_wrong() == b""


@pytest.fixture
def caches(lib):
    made = []

    def make(**kw):
        made.append(Cache(lib, **kw))
        return made[-1]
    yield make
    for c in made:
        c.close()


@pytest.mark.parametrize("mapped", (True, False))
@pytest.mark.parametrize("seed", (1, 2, 3))
def test_calls_one_after_the_other_without_waiting(lib, caches, mapped, seed):
    """Descriptors of many calls, a few KB to half a MB each, beyond both halves of the memory that they wait in."""
    rng = random.Random(seed)
    n = 600
    c = caches(seqs=n, longest=260, pages=4000, requests=n, mapped=mapped)
    waited, done = 0, dict.fromkeys(("append", "attend", "even", "read", "fork", "copy", "free", "trim", "compact"), 0)
    for step in range(700):
        what = rng.choice(("append", "append", "attend", "attend", "even", "read", "fork", "copy", "free", "trim", "compact"))
        before = lib.host_waiting()
        full = [s for s in range(n) if c.rows[s]]
        empty = [s for s in range(n) if not c.rows[s]]
        some = rng.randint(100, 400)
        if what == "append":
            st = c.append([(s, min(rng.choice((0, 1, 1, 5, 32, 70)), 260 - len(c.rows[s]))) for s in rng.sample(range(n), some)])
            assert st in (B.AIF_OK, B.AIF_ERANGE)
        elif what in ("attend", "even"):
            asks = [(rng.randrange(n), rng.choice((0, 1, 2, 8)) if what == "attend" else 1) for _ in range(some)]
            assert c.attend(asks, what == "even") == B.AIF_OK
        elif what == "read" and full:
            parts = []
            for s in rng.choices(full, k=some):
                first = rng.randrange(len(c.rows[s]))
                if None not in c.rows[s][first:]:
                    parts.append((s, first, len(c.rows[s]) - first))
            assert c.read(parts) == B.AIF_OK
        elif what in ("fork", "copy") and full and empty:
            dst = rng.sample(empty, min(len(empty), some))
            assert c.branch(what, rng.choices(full, k=len(dst)), dst) in (B.AIF_OK, B.AIF_ERANGE)
        elif what == "free" and full:
            c.free(rng.sample(full, min(len(full), some // 2)))
        elif what == "trim":
            assert c.trim(rng.sample(range(n), some), rng.choice((0, 40)), rng.choice((1, 33, 100))) == B.AIF_OK
        elif what == "compact":
            assert c.compact() == B.AIF_OK
        done[what] += 1
        waited += lib.host_waiting() < before           # a call that waited for earlier ones
    assert waited >= 4 and all(done.values()), (waited, done)
    c.check()


def _a_cache(caches, mapped=True):
    """Sequences 0..5 of 40 to 200 rows; 6 a fork of 0; scattered pages; 7..15 empty."""
    c = caches(seqs=16, longest=300, pages=60, requests=16, mapped=mapped)
    for turn in range(4):
        assert c.append([(s, 10 * (s + 1)) for s in range(6)]) == B.AIF_OK
    assert c.branch("fork", [0], [6]) == B.AIF_OK
    c.free([2])
    return c


CALLS = [("append", lambda c: c.append([(0, 5), (6, 40), (7, 90), (8, 0)]), (0, 6, 7, 8)),
         ("append of many runs", lambda c: c.append([(s, 1 + 7 * s) for s in range(15)]), tuple(range(15))),
         ("fork", lambda c: c.branch("fork", [1, 5], [7, 8]), (7, 8)), ("copy", lambda c: c.branch("copy", [1, 5], [7, 8]), (7, 8)),
         ("trim", lambda c: c.trim([5, 4, 1], 10, 40), (5, 4, 1)), ("compact", lambda c: c.compact(), tuple(range(16)))]


@pytest.mark.parametrize("error", (OUT_OF_MEMORY, LAUNCH_FAILURE))
@pytest.mark.parametrize("what,call,lost", CALLS, ids=[x[0] for x in CALLS])
def test_a_call_that_the_device_fails_leaves_what_it_changes_empty(lib, caches, what, call, lost, error):
    failed = 0
    for at in range(1, 8):
        c = _a_cache(caches)
        c.check()
        lib.host_fail(at, error)
        before = lib.host_calls()
        st = call(c)
        if lib.host_calls() < before + at:
            assert st == B.AIF_OK
            lib.host_fail(0, 0)
            c.check()
            break
        assert st == B.AIF_EDEVICE and b"as the test asked" in lib.aif_cache_last_error(c.h)
        failed += 1
        lib.host_fail(0, 0)
        for s in lost:
            assert lib.aif_cache_len(c.h, s) == 0, (s, at)
            c.rows[s] = []
        assert c.free_pages() == c.pages - sum(-(-len(c.rows[s]) // c.pl) for s in range(16) if s != 6)     # (6 has the pages of 0, or is lost as 0 is)
        assert c.append([(s, 45) for s in lost[:3]]) == B.AIF_OK       # the context goes on
        c.check()
    assert failed and at < 7


@pytest.mark.parametrize("error", (OUT_OF_MEMORY, LAUNCH_FAILURE))
def test_queries_and_reads_that_the_device_fails_change_nothing(lib, caches, error):
    for call in (lambda c: c.attend([(0, 1), (5, 3)]), lambda c: c.read([(0, 1, 20), (6, 0, 40)])):
        c = _a_cache(caches)
        lib.host_fail(1, error)
        assert call(c) == B.AIF_EDEVICE
        lib.host_fail(0, 0)
        assert call(c) == B.AIF_OK
        c.check()


def test_a_wait_for_the_descriptors_memory_that_fails(lib, caches):
    """The record and the wait between the halves of it: nothing is enqueued, and the same call goes through afterwards."""
    c = caches(seqs=400, longest=60, pages=900, requests=400)
    assert c.append([(s, 33) for s in range(400)]) == B.AIF_OK
    asks = [(s, 1 + s % 2) for s in range(400)]
    waits = 0
    while waits < 4:
        before = lib.host_waiting()
        for at in (1, 2):
            lib.host_fail(at, OUT_OF_MEMORY)
            calls = lib.host_calls()
            st = c.attend(asks[:300 + waits])
            assert lib.host_calls() >= calls + 1 and (st == B.AIF_OK) == (lib.host_calls() < calls + at)
            assert st in (B.AIF_OK, B.AIF_EDEVICE)
            lib.host_fail(0, 0)
        assert c.attend(asks) == B.AIF_OK
        waits += lib.host_waiting() < before
    c.check()
