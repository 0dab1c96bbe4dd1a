"""Cases of the paged-cache operators: tables, 8-bit append, page selection, attention.

After ``rehydrate`` has put cached chunks in place, a serving program gives the
requests their pages, keeps the rows in 8 bits and attends over them.  The
cases here are that work, from one token of one request up to a chunk prefill
over a recalled context.  A case is a dict of plain values; ``case["kind"]``:

* ``tables``  requests grow: new pages from a free list into the page tables,
              and the slot of every new token;
* ``append``  bf16 K and V rows into the 8-bit paged cache, with a power-of-two
              scale for each (page, head) and the pages' key sums;
* ``attend``  attention over the paged cache (8 bits or bf16), from one query a
              request to whole chunks;
* ``sparse``  one query a request: pages selected by their key sums, then the
              attention over the selected pages alone.

``own`` is set from outside: False computes the plain form, True calls the
library.  ``exact`` computes the definition in 64 bits.
"""

from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
E4M3_MAX = 448.0
MIN_EXP = -100           # smallest exponent of a stored scale


def _km():
    import paper_2606_23581_amd as km

    return km


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _attend(name, **kw):
    c = dict(name=name, kind="attend", requests=1, queries=1, ragged_q=False, keys=256, ragged=False, kv_heads=8,
             group=8, dim=128, page=16, cache="e4m3", causal=True, window=0, lse=False, handle=False)
    c.update(kw)
    return c


def listed():
    return [
        # one decode step of 64 requests in a serving batch: a page now and
        # then, one slot each (latency and launches count)
        dict(name="tables_step", kind="tables", requests=64, before=8000, grow=1, ragged=True, page=16, short=0,
             handle=True),
        # a batch of ragged prompts is admitted at once
        dict(name="tables_admit", kind="tables", requests=256, before=0, grow=4096, ragged=True, page=16, short=0,
             handle=False),
        # the new token's rows of 64 requests in one layer, pages mostly half full
        dict(name="append_step", kind="append", chunks=64, layers=1, heads=8, dim=128, tokens=1, before=4000,
             ragged=True, page=16, sums=True, packed=True, handle=True),
        # one prompt chunk of eight requests in one layer, ragged, larger pages
        dict(name="append_prompt", kind="append", chunks=8, layers=1, heads=8, dim=128, tokens=1024, before=4000,
             ragged=True, page=64, sums=True, packed=True, handle=False),
        # rehydrated chunks of a recall, four layers at a time, kept in 8 bits
        dict(name="append_recall", kind="append", chunks=64, layers=4, heads=8, dim=128, tokens=1024, before=0,
             ragged=False, page=16, sums=True, packed=False, handle=False),
        # first tokens after one short cached chunk: latency
        _attend("decode_short", keys=256, group=4, handle=True),
        # one request decodes over a recall of 64 chunks x 1024 tokens
        _attend("decode_recall", keys=65536, handle=True),
        # a batch of ragged requests, as a server decodes them
        _attend("decode_batch", requests=64, keys=8192, ragged=True, handle=True),
        # MHA rows in the bf16 pool that rehydrate writes, a sliding window
        _attend("decode_mha_window", requests=16, keys=8192, ragged=True, kv_heads=32, group=1, page=32,
                cache="bf16", window=4096, lse=True),
        # a prompt chunk of 1024 tokens over a recalled context, 64 query heads
        _attend("prefill_chunk", requests=1, queries=1024, keys=16384),
        # ragged prompt chunks of eight requests on the bf16 pool
        _attend("prefill_ragged", requests=8, queries=1024, ragged_q=True, keys=2048, ragged=True, kv_heads=4,
                group=7, page=64, cache="bf16", lse=True),
        # long recalls, 64 pages of 16 tokens selected for each KV head
        dict(name="sparse_recall", kind="sparse", requests=8, keys=65536, ragged=True, kv_heads=8, group=8, dim=128,
             page=16, keep=64, first=1, last=4, handle=True),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], even over its logarithm."""
    return int(min(hi, max(lo, round(float(lo) * (float(hi) / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["tables", "append", "append", "attend", "attend", "attend", "attend", "sparse"])
    page = rng.choice([16, 16, 32, 64])
    ragged = rng.random() < 0.7
    handle = rng.random() < 0.5
    if kind == "tables":
        return dict(kind=kind, requests=_log(rng, 1, 512), before=rng.choice([0, _log(rng, 1, 8000)]),
                    grow=_log(rng, 1, 2048), ragged=ragged, page=page, short=rng.choice([0, 0, 0, 3]), handle=handle)
    if kind == "append":
        c = dict(kind=kind, chunks=_log(rng, 1, 64), layers=_log(rng, 1, 4), heads=rng.choice([1, 2, 4, 8, 32]),
                 dim=rng.choice([64, 128, 128]), tokens=_log(rng, 1, 1024), before=rng.choice([0, _log(rng, 1, 4000)]),
                 ragged=ragged, page=page, sums=rng.random() < 0.7, packed=rng.random() < 0.5, handle=handle)
        while c["chunks"] * c["layers"] * c["heads"] * c["dim"] * (c["tokens"] + c["before"]) > 3 << 28:
            k = "chunks" if c["chunks"] > 1 else "layers" if c["layers"] > 1 else "before"
            c[k] = max(1, c[k] // 2)
        return c
    dim = rng.choice([64, 128, 128, 128])
    kv_heads, group = rng.choice([(8, 8), (8, 4), (4, 7), (2, 6), (1, 8), (32, 1), (1, 16), (8, 5)])
    if kind == "sparse":
        c = dict(kind=kind, requests=_log(rng, 1, 32), keys=_log(rng, 200, 65536), ragged=ragged, kv_heads=kv_heads,
                 group=group, dim=dim, page=page, keep=_log(rng, 8, 128), first=rng.choice([0, 1, 2]),
                 last=rng.choice([1, 2, 4]), handle=handle)
        while c["requests"] * c["keys"] * kv_heads * dim > 1 << 29:
            c["requests"] = max(1, c["requests"] // 2)
            if c["requests"] == 1:
                c["keys"] //= 2
        return c
    long = rng.random()
    queries = 1 if long < 0.4 else _log(rng, 2, 8) if long < 0.6 else _log(rng, 9, 1024)
    c = _attend("", requests=_log(rng, 1, 64), queries=queries, ragged_q=rng.random() < 0.5,
                keys=_log(rng, max(queries, 40), 65536 if queries < 9 else max(queries, 16384)), ragged=ragged,
                kv_heads=kv_heads, group=group, dim=dim, page=page, cache=rng.choice(["e4m3", "e4m3", "bf16"]),
                causal=rng.random() < 0.85, lse=rng.random() < 0.3, handle=handle)
    del c["name"]
    if c["causal"] and rng.random() < 0.25:
        c["window"] = _log(rng, 16, 4096)
    rows = kv_heads * group * queries
    while c["requests"] * c["keys"] * kv_heads * dim > 1 << 29 or c["requests"] * c["keys"] * rows > 1 << 30:
        if c["requests"] > 1:
            c["requests"] = max(1, c["requests"] // 2)
        else:
            c["keys"] = max(queries, c["keys"] // 2)
            if c["keys"] == queries:
                break
    return c


def _spread(n, lo, hi, ragged):
    """n lengths in [lo, hi]: all hi, or spread evenly over the range in a mixed order."""
    if not ragged or n == 1:
        return [hi] * n
    return [lo + int((hi - lo + 0.999) * ((0.5 + 0.6180339887498949 * i) % 1.0)) for i in range(n)]


def _table_lengths(case):
    before = _spread(case["requests"], case["before"] // 2, case["before"], case["ragged"])
    grow = _spread(case["requests"] + 1, (case["grow"] + 1) // 2, case["grow"], case["ragged"])[1:]
    return before, [b + g for b, g in zip(before, grow)]


def _append_lengths(case):
    before = _spread(case["chunks"], case["before"] // 2, case["before"], case["ragged"])
    tokens = _spread(case["chunks"] + 1, (case["tokens"] + 1) // 2, case["tokens"], case["ragged"])[1:]
    return before, tokens


def _key_lengths(case):
    return _spread(case["requests"], max(1, case["keys"] // 4), case["keys"], case["ragged"])


def _query_lengths(case):
    return _spread(case["requests"] + 1, (case["queries"] + 1) // 2, case["queries"], case["ragged_q"])[1:]


def _pages(tokens, page):
    return -(-tokens // page)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(shape, gen, dtype=torch.bfloat16):
    out = torch.empty(shape, dtype=dtype, device=DEV)
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 26):
        b = min(flat.numel(), a + (1 << 26))
        flat[a:b] = torch.randn(b - a, generator=gen, device=DEV)
    return out


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _tables(lengths, page, gen, width=None):
    """An injective page table [requests, width] over a pool in random order (unused entries -1), and
    the number of pool pages (one in sixteen unused)."""
    need = [_pages(n, page) for n in lengths]
    total = max(1, sum(need))
    pool = total + total // 16 + 1
    order = torch.randperm(pool, generator=gen, device=DEV).to(torch.int32)
    width = max([1, width or 0] + need)
    table = torch.full((len(lengths), width), -1, dtype=torch.int32, device=DEV)
    rows = torch.tensor([r for r, n in enumerate(need) for _ in range(n)], dtype=torch.long, device=DEV)
    cols = torch.tensor([j for n in need for j in range(n)], dtype=torch.long, device=DEV)
    table[rows, cols] = order[:sum(need)]
    return table, pool


def _cache8(pool, page, heads, dim, gen, layers=None):
    """A filled 8-bit cache: K, V as [(layers,) pages, page, heads, dim] views of a tensor that holds a
    (page, head)'s tokens together, their scales, and pages' key sums."""
    lead = () if layers is None else (layers,)
    n = len(lead)
    planes, scales = [], []
    for _ in range(2):
        x = torch.empty((*lead, pool, heads, page, dim), dtype=torch.float8_e4m3fn, device=DEV)
        bits = x.view(torch.uint8).view(-1)
        for a in range(0, bits.numel(), 1 << 26):
            b = min(bits.numel(), a + (1 << 26))
            v = torch.randn(b - a, generator=gen, device=DEV).mul_(80.0).clamp_(-E4M3_MAX, E4M3_MAX)
            bits[a:b] = v.to(torch.float8_e4m3fn).view(torch.uint8)
        planes.append(x.transpose(n + 1, n + 2))
        e = torch.randint(-8, -5, (*lead, pool, heads), generator=gen, device=DEV)
        scales.append(torch.exp2(e.float()))
    return planes, scales


def _whiten(cache, table, lengths, page):
    """NaN in the slots of a cache that no token uses, as memory holds before its first use."""
    used = torch.zeros(cache.shape[-4], page, dtype=torch.bool, device=DEV)
    n = torch.tensor(lengths, device=DEV)
    at = torch.arange(table.shape[1] * page, device=DEV).view(-1, page)
    ok = at[None] < n[:, None, None]
    pages = table.long().clamp(min=0)[:, :, None].expand_as(ok)
    inner = torch.arange(page, device=DEV).expand_as(ok)
    used[pages[ok], inner[ok]] = True
    hole = ~used
    if cache.dtype == torch.float8_e4m3fn:
        cache.view(torch.uint8).masked_fill_(hole[:, :, None, None], 0x7F)
    else:
        cache.masked_fill_(hole[:, :, None, None], float("nan"))


def prepare(case, seed):
    gen = _gen(seed)
    page, kind = case["page"], case["kind"]
    s = {"case": case, "kept": {}}
    if kind == "tables":
        before, after = _table_lengths(case)
        width = max(_pages(n, page) for n in after) + 3
        table, pool = _tables(before, page, gen, width)
        taken = torch.zeros(pool, dtype=torch.bool, device=DEV)
        taken[table[table >= 0].long()] = True
        need = sum(_pages(a, page) - _pages(b, page) for a, b in zip(after, before))
        free = max(1, need + (64 if not case["short"] else -case["short"]))
        ids = torch.arange(pool + free, device=DEV)
        ids = ids[~torch.cat([taken, torch.zeros(free, dtype=torch.bool, device=DEV)])]
        ids = ids[torch.randperm(ids.numel(), generator=gen, device=DEV)][:free + 5].to(torch.int32)
        total = sum(a - b for a, b in zip(after, before))
        s.update(before=_i32(before), after=_i32(after), table=table, free=ids.contiguous(), begin=_i32([5]),
                 end=_i32([0]), base=torch.zeros(len(after) + 1, dtype=torch.int32, device=DEV),
                 slots=torch.zeros(total + total // 8 + 3, dtype=torch.int64, device=DEV),
                 pool=pool + free, status=_i32([0]))
        return s
    if kind == "append":
        before, tokens = _append_lengths(case)
        L, H, D = case["layers"], case["heads"], case["dim"]
        table, pool = _tables([b + t for b, t in zip(before, tokens)], page, gen)
        (kc, vc), (ks, vs) = _cache8(pool, page, H, D, gen, layers=L)
        n = max(tokens)
        if case["packed"]:
            base = [sum(tokens[:c]) for c in range(len(tokens))]
            rows = _randn((L, sum(tokens), 2, H, D), gen)
            s.update(k=rows[:, :, 0], v=rows[:, :, 1], base=_i32(base), n=n)
        else:
            rows = _randn((2, case["chunks"], L, n, H, D), gen)
            s.update(k=rows[0], v=rows[1], base=None, n=n)
        s.update(before=_i32(before), tokens=_i32(tokens), table=table, pool=pool, kc=kc, vc=vc, ks=ks, vs=vs)
        if case["sums"]:
            s.update(sum=torch.zeros(L, pool, H, D, dtype=torch.int8, device=DEV),
                     sum_scale=torch.ones(L, pool, H, device=DEV))
        return s
    lengths = _key_lengths(case)
    H, G, D = case["kv_heads"], case["group"], case["dim"]
    table, pool = _tables(lengths, page, gen)
    s.update(table=table, pool=pool, kv=_i32(lengths), n_keys=max(lengths), scale=D ** -0.5)
    if case.get("cache", "e4m3") == "bf16":
        rows = _randn((pool, page, 2, H, D), gen)
        s.update(kc=rows[:, :, 0], vc=rows[:, :, 1], ks=None, vs=None)
    else:
        (kc, vc), (ks, vs) = _cache8(pool, page, H, D, gen)
        s.update(kc=kc, vc=vc, ks=ks, vs=vs)
    for c in (s["kc"], s["vc"]):
        _whiten(c, table, lengths, page)
    if kind == "sparse":
        # sums of the pages as the append makes them (of a partial last page: unused)
        x = torch.nan_to_num(s["kc"].float()).sum(1)
        e = _exp_for(x.abs().amax(-1), 127.0)
        s["sum"] = torch.round(torch.ldexp(x, -e[..., None])).to(torch.int8)
        s["sum_scale"] = torch.ldexp(s["ks"], e)
        R = case["requests"]
        s.update(q=_randn((R, H * G, D), gen), sel=torch.zeros(R, H, case["keep"], dtype=torch.int32, device=DEV),
                 count=torch.zeros(R, H, dtype=torch.int32, device=DEV))
    else:
        nq = _query_lengths(case)
        base = [sum(nq[:r]) for r in range(len(nq))]
        s.update(q=_randn((sum(nq), H * G, D), gen), nq=_i32(nq), base=_i32(base), n_queries=max(nq))
        if case["lse"]:
            s["lse"] = torch.zeros(s["q"].shape[:2], device=DEV)
    s["out"] = torch.zeros_like(s["q"])
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return _OWN[state["case"]["kind"]](state) if own else _PLAIN[state["case"]["kind"]](state)


def _call(s, name, prepare_call, direct_call):
    """A program with fixed buffers prepares a call once and launches it each step; one whose tensors
    change makes the whole call."""
    if not s["case"]["handle"]:
        return direct_call()
    if name not in s["kept"]:
        s["kept"][name] = prepare_call()
    s["kept"][name].launch()


def _own_tables(s):
    km = _km()
    a = (s["before"], s["after"], s["free"], s["table"])
    kw = dict(page_size=s["case"]["page"], n_pool_pages=s["pool"], free_begin=s["begin"], free_end=s["end"],
              token_base=s["base"], slots=s["slots"], status=s["status"])
    _call(s, "tables", lambda: km.prepare_page_tables(*a, **kw), lambda: km.page_tables(*a, **kw))
    return {"table": s["table"], "base": s["base"], "slots": s["slots"], "end": s["end"]}


def _own_append(s):
    km = _km()
    a = (s["k"], s["v"], s["kc"], s["vc"], s["ks"], s["vs"], s["table"])
    kw = dict(n_tokens=s["n"], tokens_before=s["before"], chunk_tokens=s["tokens"], row_base=s["base"],
              k_sum=s.get("sum"), k_sum_scale=s.get("sum_scale"))
    _call(s, "append", lambda: km.prepare_append_paged8(*a, **kw), lambda: km.append_paged8(*a, **kw))
    return _cache_of(s)


def _cache_of(s):
    out = {"k": s["kc"], "v": s["vc"], "k_scale": s["ks"], "v_scale": s["vs"]}
    if "sum" in s:
        out.update(sum=s["sum"], sum_scale=s["sum_scale"])
    return out


def _own_attend(s):
    km = _km()
    c = s["case"]
    a = (s["q"], s["kc"], s["vc"], s["out"], s["table"], s["kv"])
    kw = dict(n_queries=s["n_queries"], n_keys=s["n_keys"], q_base=s["base"], q_tokens=s["nq"], k_scale=s["ks"],
              v_scale=s["vs"], scale=s["scale"], causal=c["causal"], window=c["window"], lse=s.get("lse"))
    _call(s, "attend", lambda: km.prepare_attend_paged(*a, **kw), lambda: km.attend_paged(*a, **kw))
    return {"out": s["out"], "lse": s["lse"]} if c["lse"] else {"out": s["out"]}


def _own_sparse(s):
    km = _km()
    c = s["case"]
    a = (s["q"], s["sum"], s["sum_scale"], s["table"], s["kv"], s["sel"], s["count"])
    kw = dict(n_keys=s["n_keys"], page_size=c["page"], n_first=c["first"], n_last=c["last"])
    _call(s, "select", lambda: km.prepare_select_pages(*a, **kw), lambda: km.select_pages(*a, **kw))
    a2 = (s["q"], s["kc"], s["vc"], s["out"], s["table"], s["kv"])
    kw2 = dict(n_queries=1, n_keys=s["n_keys"], k_scale=s["ks"], v_scale=s["vs"], scale=s["scale"], sel=s["sel"],
               sel_count=s["count"])
    _call(s, "attend", lambda: km.prepare_attend_paged(*a2, **kw2), lambda: km.attend_paged(*a2, **kw2))
    return {"out": s["out"], "sel": s["sel"], "count": s["count"]}


_OWN = {"tables": _own_tables, "append": _own_append, "attend": _own_attend, "sparse": _own_sparse}


# ---------------------------------------------------------------------------
# plain forms, 32 bits
# ---------------------------------------------------------------------------

def _plain_tables(s):
    page, table, free = s["case"]["page"], s["table"], s["free"]
    width = table.shape[1]
    before, after = s["before"].long(), s["after"].long()
    p0, p1 = (before + page - 1) // page, (after + page - 1) // page
    take = p1 - p0
    first = torch.cumsum(take, 0) - take
    j = torch.arange(width, device=DEV)[None]
    at = s["begin"].long() + first[:, None] + j - p0[:, None]
    new = torch.where(at < free.numel(), free[at.clamp(0, free.numel() - 1)], -1)
    table.copy_(torch.where((j >= p0[:, None]) & (j < p1[:, None]), new, table))
    grown = after - before
    ends = torch.cumsum(grown, 0)
    base = torch.cat([torch.zeros_like(ends[:1]), ends])
    i = torch.arange(s["slots"].numel(), device=DEV)
    r = torch.searchsorted(ends, i, right=True).clamp(max=grown.numel() - 1)
    tok = before[r] + i - base[r]
    pg = table[r, (tok // page).clamp(0, width - 1)].long()
    slots = torch.where((i < ends[-1]) & (pg >= 0), pg * page + tok % page, -1)
    end = torch.clamp(s["begin"].long() + take.sum(), max=free.numel()).to(torch.int32)
    return {"table": table, "base": base.to(torch.int32), "slots": slots, "end": end}


def _exp_for(amax, top):
    """The least e with amax <= top * 2^e (MIN_EXP for zero and below it)."""
    m, e = torch.frexp(amax)                       # amax = m 2^e, m in [0.5, 1)
    tm, te = math.frexp(top)
    e = e - te + (m > tm).to(e.dtype)
    return torch.where(amax > 0, e, torch.full_like(e, MIN_EXP)).clamp(min=MIN_EXP)


def _plain_append(s):
    case = s["case"]
    page, table = case["page"], s["table"]
    before, tokens = s["before"].long(), s["tokens"].long()
    C, L = case["chunks"], case["layers"]
    H, D = case["heads"], case["dim"]
    n_pages = (s["n"] + page - 2) // page + 1              # pages that n tokens can touch
    j = (before // page)[:, None] + torch.arange(n_pages, device=DEV)        # [C, P] page of the request
    pos = j[:, :, None] * page + torch.arange(page, device=DEV)              # [C, P, page] token of the request
    isnew = (pos >= before[:, None, None]) & (pos < (before + tokens)[:, None, None])
    isold = pos < before[:, None, None]
    live = isnew.any(-1)                                                     # [C, P]
    pg = table[torch.arange(C, device=DEV)[:, None], j.clamp(max=table.shape[1] - 1)].long()
    row = (pos - before[:, None, None]).clamp(0, s["n"] - 1)
    cc = torch.arange(C, device=DEV)[:, None, None]
    pgl, full = pg[live], (isnew | isold).all(-1)[live]
    for rows, cache, scale in ((s["k"], s["kc"], s["ks"]), (s["v"], s["vc"], s["vs"])):
        if s["base"] is not None:
            at = (s["base"].long()[:, None, None] + row).clamp(max=rows.shape[1] - 1)
            x = rows[:, at].float()                                          # [L, C, P, page, H, D]
        else:
            x = rows[cc, :, row].float().permute(3, 0, 1, 2, 4, 5)
        x = x[:, live]                                                       # [L, N, page, H, D]
        new, old = isnew[live][None, :, :, None, None], isold[live][None, :, :, None, None]
        amax = torch.where(new & torch.isfinite(x), x.abs(), 0.0).amax((2, 4))        # [L, N, H]
        e = _exp_for(amax, E4M3_MAX)
        had, e_old = old.any(2).squeeze(-1), torch.frexp(scale[:, pgl])[1] - 1
        e = torch.where(had & (e_old > e), e_old, e)
        held = cache[:, pgl].float()
        shifted = torch.ldexp(held, torch.where(had, e_old - e, torch.zeros_like(e))[:, :, None, :, None])
        val = torch.where(new, torch.ldexp(x, -e[:, :, None, :, None]), shifted).to(torch.float8_e4m3fn)
        bits = torch.where(new | old, val.view(torch.uint8), cache.view(torch.uint8)[:, pgl])
        cache.view(torch.uint8)[:, pgl] = bits
        scale[:, pgl] = torch.ldexp(torch.ones_like(amax), e)
        if cache is s["kc"] and case["sums"]:
            t = torch.nan_to_num(val.float()).sum(2)
            es = _exp_for(t.abs().amax(-1), 127.0)
            q8 = torch.round(torch.ldexp(t, -es[..., None])).to(torch.int8)
            done = full[None, :, None]
            s["sum"][:, pgl] = torch.where(done[..., None], q8, s["sum"][:, pgl])
            s["sum_scale"][:, pgl] = torch.where(done, torch.ldexp(scale[:, pgl], es), s["sum_scale"][:, pgl])
    return _cache_of(s)


def _gathered(cache, scale, pages):
    """The rows of pages [..., n] in 32 bits: [..., n, page, heads, dim]."""
    at = pages.long().clamp(min=0)
    x = cache.view(torch.uint8)[at].view(torch.float8_e4m3fn).float() if scale is not None else cache[at].float()
    return x if scale is None else x * scale[at][..., None, :, None]


def _softmax_rows(sc, seen, v):
    """softmax(sc over the keys that a row sees) @ v, and the log of the sum; rows that see none: 0, -inf."""
    sc = torch.where(seen, sc, float("-inf"))
    m = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - torch.where(torch.isfinite(m), m, 0.0))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    return out, (torch.log(total) + m).squeeze(-1)


def _plain_attend(s):
    c = s["case"]
    H, G, D = c["kv_heads"], c["group"], c["dim"]
    R, nq, n = c["requests"], s["n_queries"], s["n_keys"]
    kv, nqs = s["kv"].long(), s["nq"].long()
    pages = s["table"][:, :_pages(n, c["page"])]
    pos = torch.arange(pages.shape[1] * c["page"], device=DEV)
    there = pos[None] < kv[:, None]                                          # [R, n]
    k = _gathered(s["kc"], s["ks"], pages).flatten(1, 2).permute(0, 2, 3, 1)           # [R, H, D, n]
    v = _gathered(s["vc"], s["vs"], pages).flatten(1, 2)
    v = torch.where(there[:, :, None, None], v, 0.0).transpose(1, 2)                   # [R, H, n, D]
    i = torch.arange(nq, device=DEV)
    at = s["base"].long()[:, None] + i
    at = torch.where(i[None] < nqs[:, None], at, s["q"].shape[0])
    q = s["q"].float()[at.clamp(max=s["q"].shape[0] - 1)]                    # [R, nq, H G, D]
    q = q.view(R, nq, H, G, D).transpose(1, 2).reshape(R, H, nq * G, D)
    sc = torch.matmul(q, k) * s["scale"]
    last = (kv - nqs)[:, None] + i if c["causal"] else (kv - 1)[:, None].expand(R, nq)
    seen = there[:, None] & (pos <= last[..., None])
    if c["window"]:
        seen = seen & (pos > last[..., None] - c["window"])
    seen = seen[:, None, :, None].expand(R, 1, nq, G, pos.numel()).reshape(R, 1, nq * G, pos.numel())
    o, lse = _softmax_rows(sc, seen, v)
    o = o.view(R, H, nq, G, D).transpose(1, 2).reshape(R, nq, H * G, D)
    out = torch.zeros(s["q"].shape[0] + 1, H * G, D, device=DEV)
    out[at] = o
    got = {"out": out[:-1].to(torch.bfloat16)}
    if c["lse"]:
        flat = torch.zeros(s["q"].shape[0] + 1, H * G, device=DEV)
        flat[at] = lse.view(R, H, nq, G).transpose(1, 2).reshape(R, nq, H * G)
        got["lse"] = flat[:-1]
    return got


def _plain_sparse(s):
    c = s["case"]
    H, G, D, page = c["kv_heads"], c["group"], c["dim"], c["page"]
    R, keep = c["requests"], c["keep"]
    kv = s["kv"].long()
    pages = s["table"].long().clamp(min=0)
    n = (kv + page - 1) // page
    q = s["q"].float().view(R, H, G, D)
    e = _exp_for(q.abs().amax((2, 3)), 127.0)
    q8 = torch.round(torch.ldexp(q, -e[:, :, None, None]))
    dots = torch.matmul(q8, s["sum"][pages].float().permute(0, 2, 3, 1))     # [R, H, G, P]
    score = dots.amax(2) * s["sum_scale"][pages].transpose(1, 2)
    j = torch.arange(pages.shape[1], device=DEV)
    always = (j < c["first"]) | (j >= (n - c["last"])[:, None])
    score = torch.where(always[:, None], float("inf"), score)
    score = torch.where((j < n[:, None])[:, None], score, float("-inf"))
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :keep]
    count = torch.clamp(n, max=keep)[:, None].expand(R, H)
    k_ = torch.arange(order.shape[-1], device=DEV)
    order = torch.where(k_ < count[..., None], order, pages.shape[1])
    order = torch.sort(order, dim=-1).values
    sel = torch.full((R, H, keep), -1, dtype=torch.int32, device=DEV)
    sel[..., :order.shape[-1]] = torch.where(order < pages.shape[1], order, -1)
    # attention over the selected pages
    got = order.clamp(max=pages.shape[1] - 1)
    pg = torch.gather(pages[:, None].expand(R, H, -1), 2, got)
    h = torch.arange(H, device=DEV)[None, :, None]
    k = s["kc"].view(torch.uint8)[pg, :, h].view(torch.float8_e4m3fn).float() * s["ks"][pg, h][..., None, None]
    v = s["vc"].view(torch.uint8)[pg, :, h].view(torch.float8_e4m3fn).float() * s["vs"][pg, h][..., None, None]
    pos = order[..., None] * page + torch.arange(page, device=DEV)
    seen = (pos < kv[:, None, None, None]).flatten(2)
    v = torch.where(seen[..., None], v.flatten(2, 3), 0.0)
    sc = torch.matmul(q, k.flatten(2, 3).transpose(2, 3)) * s["scale"]
    o, _ = _softmax_rows(sc, seen[:, :, None], v)
    return {"out": o.reshape(R, H * G, D).to(torch.bfloat16), "sel": sel, "count": count.to(torch.int32)}


_PLAIN = {"tables": _plain_tables, "append": _plain_append, "attend": _plain_attend, "sparse": _plain_sparse}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def _visible(case, n, nq):
    """(keys that some query of a request sees, the sum over its queries of the keys each sees)."""
    if not case["causal"]:
        return n, n * nq
    w = case["window"] or n + nq
    total, low = 0, n
    for i in range(nq):
        top = n - nq + i + 1                       # keys [max(0, top - w), top)
        if top > 0:
            low = min(low, max(0, top - w))
            total += top - max(0, top - w)
    return n - low, total


def work(case):
    kind, page = case["kind"], case["page"]
    if kind == "tables":
        before, after = _table_lengths(case)
        new = sum(_pages(a, page) - _pages(b, page) for a, b in zip(after, before))
        tokens = sum(a - b for a, b in zip(after, before))
        slots = tokens + tokens // 8 + 3
        return {"bytes": 4.0 * (3 * len(before) + 2 * new + 3) + 8.0 * slots, "flops": 0.0}
    if kind == "append":
        before, tokens = _append_lengths(case)
        units = 2 * case["layers"] * case["heads"]
        touched = sum(_pages(b + t, page) - b // page for b, t in zip(before, tokens))
        full = sum((b + t) // page - b // page for b, t in zip(before, tokens))
        got = units * case["dim"] * sum(tokens) * 3.0 + units * 4.0 * touched
        if case["sums"]:
            # a page that fills up: its older keys read, its sums written
            held = sum(b % page for b, t in zip(before, tokens) if (b + t) // page > b // page)
            got += units / 2 * (full * (case["dim"] + 4.0) + held * case["dim"])
        return {"bytes": got, "flops": 0.0}
    H, G, D = case["kv_heads"], case["group"], case["dim"]
    lengths = _key_lengths(case)
    if kind == "sparse":
        n = [_pages(t, page) for t in lengths]
        kept = sum(min(case["keep"], p) for p in n)
        return {"bytes": H * (sum(n) * (D + 4.0) + kept * (page * D * 2.0 + 12.0))
                + 4.0 * case["requests"] * H * G * D + 4.0 * sum(n),
                "flops": 2.0 * H * G * D * (sum(n) + 2 * kept * page)}
    nq = _query_lengths(case)
    el = 2 if case["cache"] == "bf16" else 1
    keys = pairs = 0
    for n, m in zip(lengths, nq):
        a, b = _visible(case, n, m)
        keys, pairs = keys + a, pairs + b
    got = 2.0 * el * H * D * keys + 4.0 * sum(nq) * H * G * D + 4.0 * keys / page
    if el == 1:
        got += 8.0 * H * keys / page
    if case["lse"]:
        got += 4.0 * sum(nq) * H * G
    return {"bytes": got, "flops": 4.0 * H * G * D * pairs}


# ---------------------------------------------------------------------------
# the definition, 64 bits
# ---------------------------------------------------------------------------

def _rows64(cache, scale, pages, n, h):
    x = cache[:, :, h].contiguous().view(torch.uint8 if scale is not None else torch.bfloat16)[pages.long()]
    if scale is None:
        return x.double().flatten(0, 1)[:n]
    x = x.view(torch.float8_e4m3fn).double()
    return (x * scale[pages.long(), h].double()[:, None, None]).flatten(0, 1)[:n]


def _attend64(q, k, v, scale, low, top):
    """Rows q [m, D] over keys [low[i], top[i]) of k, v."""
    z = torch.matmul(q, k.t().contiguous()) * scale
    j = torch.arange(k.shape[0], device=DEV)
    hide = (j[None] >= top[:, None]) | (j[None] < low[:, None])
    z.masked_fill_(hide, -math.inf)
    lse = torch.logsumexp(z, -1)
    w = torch.exp(z - torch.where(torch.isinf(lse), 0.0, lse)[:, None])
    return torch.matmul(w, v), lse


def exact(case, seed):
    kind = case["kind"]
    s = prepare(case, seed)
    if kind == "tables":
        return None
    if kind == "append":
        return _exact_append(case, s)
    H, G, D, page = case["kv_heads"], case["group"], case["dim"], case["page"]
    lengths = _key_lengths(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    if kind == "sparse":
        got = _plain_sparse(s)["sel"].tolist()     # whole numbers, compared as such
        for r, n in enumerate(lengths):
            for h in range(H):
                pick = torch.tensor([p for p in got[r][h] if p >= 0], device=DEV)
                at = (pick[:, None] * page + torch.arange(page, device=DEV)).flatten()
                at = at[at < n]
                k = _rows64(s["kc"], s["ks"], s["table"][r, :_pages(n, page)], n, h)[at]
                v = _rows64(s["vc"], s["vs"], s["table"][r, :_pages(n, page)], n, h)[at]
                q = s["q"][r, h * G:(h + 1) * G].double()
                lo = torch.zeros(G, device=DEV)
                out[r, h * G:(h + 1) * G] = _attend64(q, k, v, s["scale"], lo, lo + at.numel())[0]
        return {"out": out, "sel": None, "count": None}
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device=DEV)
    nq, at = _query_lengths(case), 0
    if sum(n * m for n, m in zip(lengths, nq)) * H * G > 4 << 30:
        return None
    for r, (n, m) in enumerate(zip(lengths, nq)):
        i = torch.arange(m, device=DEV)
        top = (n - m + 1 + i) if case["causal"] else torch.full_like(i, n)
        low = (top - case["window"]).clamp(min=0) if case["window"] else torch.zeros_like(top)
        pages = s["table"][r, :_pages(n, page)]
        for h in range(H):
            k, v = _rows64(s["kc"], s["ks"], pages, n, h), _rows64(s["vc"], s["vs"], pages, n, h)
            for g in range(h * G, (h + 1) * G):
                out[at:at + m, g], lse[at:at + m, g] = _attend64(s["q"][at:at + m, g].double(), k, v, s["scale"], low,
                                                                 top)
        at += m
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def _round8(x):
    """x to the nearest e4m3 value, ties to even, as numbers in 64 bits."""
    _, e = torch.frexp(x)
    step = torch.exp2((e - 4).clamp(min=-9).double())
    return torch.round(x / step) * step


def _exact_append(case, s):
    before, tokens = _append_lengths(case)
    page, L, H = case["page"], case["layers"], case["heads"]
    if L * H * case["dim"] * (sum(tokens) + len(tokens) * page) > 1 << 29 or sum(_pages(t, page) for t in tokens) > 4096:
        return None
    got = {"k": s["kc"].double(), "v": s["vc"].double(), "k_scale": s["ks"].double(), "v_scale": s["vs"].double()}
    table = s["table"].tolist()
    for c, (b, t) in enumerate(zip(before, tokens)):
        for j in range(b // page, _pages(b + t, page)):
            lo, hi = max(b, j * page), min(b + t, (j + 1) * page)
            pg = table[c][j]
            for name, rows in (("k", s["k"]), ("v", s["v"])):
                first = (0 if s["base"] is None else sum(tokens[:c])) + lo - b
                x = (rows[c] if s["base"] is None else rows)[:, first:first + hi - lo].double()      # [L, t, H, D]
                top = x.abs().amax((1, 3))
                e = torch.ceil(torch.log2(top / E4M3_MAX)).clamp(min=MIN_EXP)
                e = e + (top > E4M3_MAX * torch.exp2(e)).double() - (top <= E4M3_MAX * torch.exp2(e - 1)).double()
                held = lo - j * page
                if held:
                    old = torch.log2(got[name + "_scale"][:, pg])
                    e = torch.maximum(e, old)
                    ratio = torch.exp2(old - e)[:, None, :, None]
                    got[name][:, pg, :held] = _round8(got[name][:, pg, :held] * ratio)
                got[name][:, pg, held:held + hi - lo] = _round8(x * torch.exp2(-e)[:, None, :, None])
                got[name + "_scale"][:, pg] = torch.exp2(e)
    if case["sums"]:
        got.update(sum=None, sum_scale=None)
    return got
