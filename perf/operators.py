"""Timed cases of the user cache: behaviour sequences held in pages of 4 bits, and what reads and moves them.

A cache holds, per user and behaviour, a key and a value row of ``kv_heads`` heads of ``d_head`` features.  A head's
features are cut into blocks of 32 (the last one shorter); a block is a power of two and signed codes of the magnitudes
0, 1/2, 1, 3/2, 2, 3, 4, 6.  Rows lie in pages, and a table names the pages of each user.

kinds of cases
  attend   queries (candidates, or the one next behaviour) over the whole of their user's cache
  window   the same where a query at position p sees the last ``window`` behaviours up to p and the first ``sinks``
  append   whole histories enter the cache and are read back as the values they stand for
  pages    a branch of every user: fork, append, copy, free, compact, read, free
"""
import math

import torch

own = False

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(name, kind, dtype, users, length, kv_heads, heads, d_head, page, queries=0, ragged=False, window=0, sinks=0,
          positions=False, rows=0):
    return {"name": name, "kind": kind, "dtype": dtype, "users": users, "length": length, "kv_heads": kv_heads, "heads": heads,
            "d_head": d_head, "page": page, "queries": queries, "ragged": ragged, "window": window, "sinks": sinks,
            "positions": positions, "rows": rows}


def listed():
    return [
        # the shortest call: one user, one next behaviour, one page
        _case("attend f32 one query", "attend", "f32", 1, 50, 1, 1, 32, 64, queries=1),
        # next-behaviour step of many users at once, shared key heads, ragged histories
        _case("attend one query 64 users", "attend", "bf16", 64, 4096, 2, 8, 128, 64, queries=1, ragged=True),
        # life-long histories, few users: the cache is all there is to read
        _case("attend one query long", "attend", "bf16", 16, 131072, 4, 16, 128, 128, queries=1),
        # a mini-batch of candidates in fp32, heads of 32, ragged histories
        _case("attend f32 candidates", "attend", "f32", 16, 333, 2, 2, 32, 64, queries=1000, ragged=True),
        # pre-ranking: 64 users x 10^4 candidates over 500 behaviours, one head of 64
        _case("attend candidates", "attend", "bf16", 64, 500, 1, 1, 64, 64, queries=10000),
        # the wide model's attention: eight heads of 16 over 2,000 behaviours
        _case("attend candidates 8 heads", "attend", "bf16", 8, 2000, 8, 8, 16, 128, queries=10000),
        # replay of logged impressions: each sees what was recent when it was shown
        _case("window impressions", "window", "bf16", 8, 20000, 2, 4, 64, 64, queries=2000, ragged=True, window=512, sinks=16, positions=True),
        # the next behaviour of many users, of whose long histories only a window counts
        _case("window one query", "window", "bf16", 128, 32768, 2, 8, 128, 64, queries=1, ragged=True, window=1024, sinks=4),
        # a short fp32 replay of odd sizes
        _case("window f32 odd", "window", "f32", 3, 777, 1, 3, 40, 32, queries=61, ragged=True, window=100, sinks=5, positions=True),
        # what the user network leaves for 64 users goes into the cache
        _case("append 64 users", "append", "bf16", 64, 500, 1, 1, 64, 64, ragged=True),
        # long fp32 histories at once
        _case("append f32 long", "append", "f32", 16, 20011, 2, 2, 128, 128),
        # what-if branches of 32 users, eight more behaviours each
        _case("pages branches", "pages", "bf16", 32, 4096, 2, 2, 128, 64, ragged=True, rows=8),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(("attend", "attend", "window", "window", "append", "pages"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    kv_heads = rng.choice((1, 1, 2, 4, 8))
    group = rng.choice((1, 1, 2, 3, 4, 8))
    d_head = rng.choice((16, 24, 32, 40, 64, 64, 80, 96, 128, 128, 192, 256))
    page = rng.choice((32, 64, 128))
    width = kv_heads * d_head
    length = _log_int(rng, 1, 65536)
    most = 400_000_000 if kind in ("attend", "window") else 60_000_000      # features held
    length = min(length, most // width)
    users = _log_int(rng, 1, max(1, min(256, most // (length * width))))
    case = _case("", kind, dtype, users, length, kv_heads, kv_heads * group, d_head, page, ragged=rng.random() < 0.6)
    del case["name"]
    if kind in ("attend", "window"):
        # scores that the plain form holds at once, their products, and rows of the outputs
        heads = users * kv_heads * group
        most = min(1_200_000_000 // (heads * length), 20_000_000_000 // (heads * length * d_head), 100_000_000 // (heads * d_head))
        case["queries"] = 1 if rng.random() < 0.35 else _log_int(rng, 1, max(1, min(10000, most)))
    if kind == "window":
        case["window"] = _log_int(rng, 1, max(1, length))
        case["sinks"] = rng.choice((0, 1, 4, 16, 64))
        case["positions"] = case["queries"] > 1 and rng.random() < 0.7
    if kind == "pages":
        case["rows"] = _log_int(rng, 1, 200)
    return case


def _lengths(case):
    """Behaviours of each user: the case's length, or spread between a fifth of it and all of it."""
    n, most = case["users"], case["length"]
    if not case["ragged"]:
        return [most] * n
    return [most if i == 0 else max(1, int(most * (0.2 + 0.8 * ((i * 0.6180339887) % 1.0)))) for i in range(n)]


def _torch_dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _rows(case, n, gen):
    """Keys and values [n, kv_heads, d_head]: features of unlike spread, as learnt projections have them."""
    shape = (n, case["kv_heads"], case["d_head"])
    spread = torch.exp(0.5 * torch.randn(shape[1:], generator=gen, device="cuda"))
    keys = torch.randn(shape, generator=gen, device="cuda") * spread
    vals = torch.randn(shape, generator=gen, device="cuda") * 0.5
    return keys.to(_torch_dtype(case)), vals.to(_torch_dtype(case))


def _inputs(case, seed):
    """What the case is made of, from the seed alone: histories one after the other, queries, positions, appended rows."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lens = _lengths(case)
    keys, vals = _rows(case, sum(lens), gen)
    x = {"lens": lens, "keys": keys, "vals": vals}
    n_q, users = case["queries"], case["users"]
    if n_q:
        x["q"] = torch.randn((users, n_q, case["heads"], case["d_head"]), generator=gen, device="cuda").to(_torch_dtype(case))
    if case["positions"]:
        at = (torch.arange(n_q, device="cuda") + torch.rand((users, n_q), generator=gen, device="cuda")) / n_q
        x["pos"] = (at * torch.tensor(lens, device="cuda")[:, None]).to(torch.int32).clamp_(min=0)
    if case["rows"]:
        x["new_keys"], x["new_vals"] = _rows(case, users * case["rows"], gen)
    return x


# ---- plain form: codes and scales in pages -------------------------------------------------------------------------
def _cut(x):
    """[..., d] as blocks of 32, zeros past its end: [..., blocks, 32] in 32 bits."""
    d = x.shape[-1]
    blocks = -(-d // 32)
    return torch.nn.functional.pad(x.float(), (0, blocks * 32 - d)).unflatten(-1, (blocks, 32))


def _encode(x):
    """Two codes a byte [..., blocks, 16] and scale bytes [..., blocks]."""
    b = _cut(x)
    most = b.abs().amax(-1)
    mant, exp = torch.frexp(most)                   # most = mant 2^exp, mant in [1/2, 1): most <= 6 2^e
    e = torch.where(mant <= 0.75, exp - 3, exp - 2).clamp_(min=-125)
    a = torch.ldexp(b.abs(), -e[..., None])
    code = torch.where(a < 2, torch.round(2 * a), torch.where(a < 4, torch.round(a) + 2, torch.round(0.5 * a) + 4))
    code = (code + 8 * (b < 0)).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _decode(codes, scales, d):
    """What codes and scales stand for, [..., d] in 32 bits."""
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=codes.device)
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    v = torch.ldexp(table[code.int()], (scales.int() - 127)[..., None])
    return v.flatten(-2)[..., :d]


def _plan(lens, page, first_page=0):
    """Page table [users, pages] and the places (page * page_len + row) of all behaviours, users one after the other."""
    width = max(1, max(-(-n // page) for n in lens))
    ln = torch.tensor(lens, device="cuda")
    count = (ln + page - 1) // page
    start = first_page + torch.cumsum(count, 0) - count
    table = start[:, None] + torch.arange(width, device="cuda")
    user = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), ln)
    pos = torch.arange(int(ln.sum()), device="cuda") - (torch.cumsum(ln, 0) - ln)[user]
    return table, table[user, pos // page] * page + pos % page, int(count.sum()), user, pos


def _write(pool, places, keys, vals):
    for name, x in (("k", keys), ("v", vals)):
        codes, scales = _encode(x)
        pool[name].flatten(0, 1)[places] = codes
        pool[name + "s"].flatten(0, 1)[places] = scales


def _read(pool, places, case):
    return [_decode(pool[n].flatten(0, 1)[places], pool[n + "s"].flatten(0, 1)[places], case["d_head"]).to(_torch_dtype(case))
            for n in ("k", "v")]


def _pool(case, n_pages):
    blocks = -(-case["d_head"] // 32)
    shape = (n_pages, case["page"], case["kv_heads"], blocks)
    make = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    return {"k": make(*shape, 16), "v": make(*shape, 16), "ks": make(*shape), "vs": make(*shape)}


def _attend(case, pool, table, lens, q, pos):
    page, d, group = case["page"], case["d_head"], case["heads"] // case["kv_heads"]
    users, n_q = q.shape[:2]
    width = table.shape[1] * page
    table = table.clamp(max=pool["k"].shape[0] - 1)
    dense = [_decode(pool[n][table], pool[n + "s"][table], d).reshape(users, width, case["kv_heads"], d).transpose(1, 2).contiguous()
             for n in ("k", "v")]                                                             # [users, kv_heads, width, d]
    rows = q.float().unflatten(2, (case["kv_heads"], group)).permute(0, 2, 1, 3, 4).reshape(users, case["kv_heads"], n_q * group, d)
    s = rows @ dense[0].transpose(2, 3) * d ** -0.5                                           # [users, kv_heads, n_q * group, width]
    j = torch.arange(width, device=q.device)
    p = (lens[:, None] - 1).expand(users, n_q) if pos is None else pos.long()
    p = p.repeat_interleave(group, 1)[:, :, None]
    see = (j < lens[:, None, None]) & (j <= p)
    if case["window"]:
        see = see & ((j > p - case["window"]) | (j < case["sinks"]))
    s = s.masked_fill_(~see[:, None], -math.inf)
    most = s.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    w = torch.exp_(s.sub_(most))
    total = w.sum(-1, keepdim=True)
    o = (w @ dense[1]) / torch.where(total > 0, total, 1.0)
    lse = (torch.log(total) + most).squeeze(-1)
    back = lambda x: x.unflatten(2, (n_q, group)).transpose(1, 2).flatten(2, 3)  # noqa: E731
    return [back(o).to(q.dtype), back(lse)]


# ---- states ---------------------------------------------------------------------------------------------------------
def _handle(case, x):
    """The framework's cache, its requests packed once, and the buffers they write."""
    from paper_2511_12934_amd import binding as B

    users, lens, rows = case["users"], x["lens"], case["rows"]
    dtype = B.AIF_F32 if case["dtype"] == "f32" else B.AIF_BF16
    pages = sum(-(-n // case["page"]) for n in lens)
    n_pages = pages
    if case["kind"] == "pages":                     # the parents, what their children append, and whole copies of the children
        more = sum(-(-(n + rows) // case["page"]) for n in lens)
        n_pages = pages + (more - pages + users) + more
    shape = dict(dtype=dtype, n_heads=case["heads"], n_kv_heads=case["kv_heads"], d_head=case["d_head"], page_len=case["page"])
    pool = torch.empty(n_pages * B.cache_page_bytes(**shape), dtype=torch.uint8, device="cuda")
    ctx = B.CacheContext(pool=pool, max_seqs=3 * users, max_len=max(lens) + rows, max_requests=users, max_queries=max(1, case["queries"]), **shape)
    starts = [0]
    for n in lens:
        starts.append(starts[-1] + n)
    st = {"ctx": ctx, "pool": pool}
    st["fill"] = [B.CacheAppend(u, x["keys"][starts[u]:starts[u + 1]], x["vals"][starts[u]:starts[u + 1]]) for u in range(users)]
    st["fill_packed"] = B.pack_cache_appends(st["fill"])
    if case["kind"] != "append":
        ctx.aif_cache_append(st["fill"], packed=st["fill_packed"])
        torch.cuda.synchronize()
        del st["fill"], st["fill_packed"]
    if case["queries"]:
        st["out"] = torch.empty_like(x["q"])
        st["lse"] = torch.empty(x["q"].shape[:3], dtype=torch.float32, device="cuda")
        st["asks"] = [B.CacheQuery(u, x["q"][u], st["out"][u], lse=st["lse"][u], positions=x["pos"][u] if case["positions"] else None,
                                   sinks=case["sinks"], window=case["window"]) for u in range(users)]
        st["asks_packed"] = B.pack_cache_queries(st["asks"])
        return st
    at = [0]
    for n in lens:
        at.append(at[-1] + n + rows)
    of = 0 if case["kind"] == "append" else 2 * users
    st["k_out"], st["v_out"] = (torch.empty((at[-1], case["kv_heads"], case["d_head"]), dtype=_torch_dtype(case), device="cuda") for _ in range(2))
    st["reads"] = [B.CacheRead(of + u, st["k_out"][at[u]:at[u + 1]], st["v_out"][at[u]:at[u + 1]]) for u in range(users)]
    st["reads_packed"] = B.pack_cache_reads(st["reads"])
    if rows:
        st["parents"], st["children"], st["copies"] = (B.cache_ids(range(k * users, (k + 1) * users)) for k in range(3))
        st["news"] = [B.CacheAppend(users + u, x["new_keys"][u * rows:(u + 1) * rows], x["new_vals"][u * rows:(u + 1) * rows])
                      for u in range(users)]
        st["news_packed"] = B.pack_cache_appends(st["news"])
    else:
        st["seqs"] = B.cache_ids(range(users))
    return st


def prepare(case, seed):
    x = _inputs(case, seed)
    st = {"case": case, "x": x}
    if own:
        st.update(_handle(case, x))
    else:
        lens, page = x["lens"], case["page"]
        st["lens"] = torch.tensor(lens, device="cuda")
        st["table"], st["places"], used, user, pos = _plan(lens, page)
        if case["kind"] == "pages":
            longer = [n + case["rows"] for n in lens]
            st["user"], st["pos"] = user, pos
            st["copy_table"], st["copy_places"], copied, u2, p2 = _plan(longer, page, used + sum(-(-m // page) - n // page for m, n in zip(longer, lens)))
            st["is_new"] = p2 >= st["lens"][u2]
            fresh, st["fresh_places"], _, fu, fp = _plan([m - n // page * page for m, n in zip(longer, lens)], page, used)
            st["fresh"], st["whole"] = fresh, st["lens"] // page       # a child: its parent's whole pages, then pages of its own
            st["total"] = used + sum(-(-m // page) - n // page for m, n in zip(longer, lens)) + copied
            st["u2"], st["p2"] = u2, p2
            used = st["total"]
        st["pool"] = _pool(case, used)
        _write(st["pool"], st["places"], x["keys"], x["vals"])
    if case["kind"] != "append":
        del x["keys"], x["vals"]                    # they are in the cache
    return st


def _branches(st):
    """Plain form of a branch of every user: the child's own pages, a copy of all of it, the copy moved down, its values."""
    case, pool, page, x = st["case"], st["pool"], st["case"]["page"], st["x"]
    lens, whole, table, fresh = st["lens"], st["whole"], st["table"], st["fresh"]
    users = torch.arange(case["users"], device=lens.device)
    # fork: the child's table is its parent's, its last page its own once it is written to
    width = st["copy_table"].shape[1]
    cols = torch.arange(width, device=lens.device)
    padded = torch.nn.functional.pad(table, (0, width - table.shape[1]))
    child = torch.where(cols < whole[:, None], padded, fresh[users[:, None], (cols - whole[:, None]).clamp(0, fresh.shape[1] - 1)])
    last = (lens % page > 0).nonzero().flatten()
    for name in pool:
        pool[name][child[last, whole[last]]] = pool[name][table[last, whole[last]]]
    u, p = st["u2"][st["is_new"]], st["p2"][st["is_new"]]
    _write(pool, child[u, p // page] * page + p % page, x["new_keys"], x["new_vals"])
    # copy: pages of its own for everything
    have = cols < ((lens + case["rows"] + page - 1) // page)[:, None]
    src, dst = child[have], st["copy_table"][have]
    for name in pool:
        pool[name][dst] = pool[name][src]
    # free the children and compact: the copies move down into the pages that they leave
    first = int(case_pages(case))
    move = torch.arange(dst.numel(), device=dst.device) + first
    for name in pool:
        pool[name][move] = pool[name][dst]          # the right side is whole before the left is written
    return _read(pool, (st["copy_places"] // page - dst.min() + first) * page + st["copy_places"] % page, case)


def case_pages(case):
    return sum(-(-n // case["page"]) for n in _lengths(case))


def run(state):
    case, x = state["case"], state["x"]
    if own:
        ctx = state["ctx"]
        if case["kind"] in ("attend", "window"):
            ctx.aif_cache_attend(state["asks"], packed=state["asks_packed"])
            return [state["out"], state["lse"]]
        if case["kind"] == "append":
            ctx.aif_cache_free(state["seqs"])
            ctx.aif_cache_append(state["fill"], packed=state["fill_packed"])
            ctx.aif_cache_read(state["reads"], packed=state["reads_packed"])
            return [state["k_out"], state["v_out"]]
        ctx.aif_cache_fork(state["parents"], state["children"])
        ctx.aif_cache_append(state["news"], packed=state["news_packed"])
        ctx.aif_cache_copy(state["children"], state["copies"])
        ctx.aif_cache_free(state["children"])
        ctx.aif_cache_compact()
        ctx.aif_cache_read(state["reads"], packed=state["reads_packed"])
        ctx.aif_cache_free(state["copies"])
        return [state["k_out"], state["v_out"]]
    if case["kind"] in ("attend", "window"):
        return _attend(case, state["pool"], state["table"], state["lens"], x["q"], x.get("pos"))
    if case["kind"] == "append":
        _write(state["pool"], state["places"], x["keys"], x["vals"])
        return _read(state["pool"], state["places"], case)
    return _branches(state)


def work(case):
    lens, kv, d, h = _lengths(case), case["kv_heads"], case["d_head"], case["heads"]
    esz = 4 if case["dtype"] == "f32" else 2
    held = kv * (d + 2 * -(-d // 32))               # a behaviour's key and value in 4 bits, with their scales
    plain = 2 * kv * d * esz
    if case["kind"] in ("attend", "window"):
        n_q, w, s = case["queries"], case["window"], case["sinks"]
        pairs = seen = 0
        for n in lens:
            if case["positions"]:
                step = max(1, n_q // 64)
                at = [int((i + 0.5) * n / n_q) for i in range(0, n_q, step)]
                each = [min(p + 1, w + min(s, max(0, p + 1 - w))) for p in at]
                pairs += int(n_q * sum(each) / len(each))
                seen += min(n, n_q * w + s)
            else:
                one = min(n, w + min(s, max(0, n - w))) if w else n
                pairs, seen = pairs + n_q * one, seen + one
        rows = case["users"] * n_q * h
        return {"bytes": seen * held + rows * (2 * d * esz + 4), "flops": 4.0 * pairs * h * d}
    if case["kind"] == "append":
        return {"bytes": 2 * sum(lens) * (plain + held), "flops": 0}
    total = sum(lens) + case["users"] * case["rows"]
    return {"bytes": total * (3 * held + plain) + case["users"] * case["rows"] * (plain + held), "flops": 0}


# ---- from the definition, in 64 bits -------------------------------------------------------------------------------
def _held(x):
    """What is left of rows [n, heads, d] once they are held in 4 bits, in 64 bits."""
    out = torch.zeros_like(x, dtype=torch.float64)
    passed = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))   # (border, the border itself rounds up)
    steps = (0.5, 0.5, 0.5, 0.5, 1.0, 1.0, 2.0)
    for lo in range(0, x.shape[-1], 32):
        b = x[..., lo:lo + 32].double()
        top = b.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 6.0))
        unit = torch.exp2(torch.where(top > 0, e, -125.0).clamp(min=-125.0))
        a, m = b.abs() / unit, torch.zeros_like(b)
        for (border, up), step in zip(passed, steps):
            m = m + step * ((a >= border) if up else (a > border))
        out[..., lo:lo + 32] = torch.sign(b) * m * unit
    return out


def exact(case, seed):
    if case["users"] * case["length"] * case["kv_heads"] * case["d_head"] > 1.5e9:
        return None
    x = _inputs(case, seed)
    lens, users = x["lens"], case["users"]
    keys, vals = _held(x["keys"]), _held(x["vals"])
    if case["kind"] == "append":
        return [keys, vals]
    starts = [0]
    for n in lens:
        starts.append(starts[-1] + n)
    if case["kind"] == "pages":
        more = [_held(x["new_keys"]), _held(x["new_vals"])]
        r = case["rows"]
        return [torch.cat([t for u in range(users) for t in (old[starts[u]:starts[u + 1]], new[u * r:(u + 1) * r])])
                for old, new in zip((keys, vals), more)]
    if 4 * users * case["queries"] * case["heads"] * case["length"] * case["d_head"] > 2e13:
        return None
    n_q, heads, d, group = case["queries"], case["heads"], case["d_head"], case["heads"] // case["kv_heads"]
    out = torch.zeros((users, n_q, heads, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((users, n_q, heads), dtype=torch.float64, device="cuda")
    for u in range(users):
        n = lens[u]
        p = x["pos"][u].long() if case["positions"] else torch.full((n_q,), n - 1, device="cuda")
        j = torch.arange(n, device="cuda")
        hidden = j[None, :] > p[:, None]
        if case["window"]:
            hidden |= (p[:, None] - j[None, :] >= case["window"]) & (j[None, :] >= case["sinks"])
        for h in range(heads):
            k, v = keys[starts[u]:starts[u + 1], h // group], vals[starts[u]:starts[u + 1], h // group]
            for lo in range(0, n_q, 1 << 12):
                at = slice(lo, min(n_q, lo + (1 << 12)))
                s = (x["q"][u, at, h].double() @ k.T.contiguous() / math.sqrt(d)).masked_fill(hidden[at], -math.inf)
                z = torch.logsumexp(s, -1)
                lse[u, at, h] = z
                out[u, at, h] = torch.exp(s - z[:, None]) @ v
    return [out, lse]
