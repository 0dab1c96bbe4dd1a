"""Cases of serving from a paged latent cache: rotated append, per-head products, attention in both forms.

``rehydrate`` puts rows of a latent and a rope key (512 + 64 columns, one row a
token for all heads) into the paged pool.  The cases here are what a program
does from there on, from one token of one request up to prompt chunks over a
recalled context; ``case["kind"]``:

* ``append``    rows of new tokens into the paged pool with their rotary
                positions applied on the way, their queries' bands with them
* ``project``   a product with a matrix of its own for every head: queries into
                the latent's columns, attention results out of them
* ``expand``    keys and values of every head from the latents in the pool
* ``latent``    attention over the pool's rows themselves (the absorbed form)
* ``expanded``  attention over expanded keys and values, with the rope keys read
                from the pool

``own`` is set from outside: False computes the plain form, True calls the
library.  ``exact`` computes the definition in 64 bits.
"""

from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
ROPE = 64                # columns of the rope key behind a latent


def _km():
    import paper_2606_23581_amd as km

    return km


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _append(name, **kw):
    c = dict(name=name, kind="append", chunks=1, tokens=1, before=0, ragged=False, page=16, rows="latent", heads=1,
             dim=576, q_heads=16, rope_dim=64, pairing="interleaved", sections=False, scaling="none", handle=False)
    c.update(kw)
    return c


def _latent(name, **kw):
    c = dict(name=name, kind="latent", requests=1, queries=1, ragged_q=False, keys=256, ragged=False, heads=16,
             latent=512, page=16, causal=True, window=0, lse=False, handle=False)
    c.update(kw)
    return c


def _expanded(name, **kw):
    c = dict(name=name, kind="expanded", requests=1, queries=256, ragged_q=False, keys=256, ragged=False, heads=16,
             dim=128, page=16, causal=True, window=0, lse=False, handle=False)
    c.update(kw)
    return c


def listed():
    return [
        # the new token of each of 64 requests in one layer: one latent row, the
        # rope bands of 16 query heads (latency and launches count)
        _append("append_step", chunks=64, before=8000, ragged=True, handle=True),
        # ragged prompts of eight requests in one layer of grouped K and V rows,
        # positions scaled for a long context
        _append("append_prompt", chunks=8, tokens=1024, before=4000, ragged=True, page=64, rows="kv", heads=8, dim=128,
                q_heads=64, rope_dim=128, pairing="neox", scaling="pairs"),
        # a decode step's queries into the latent's columns
        dict(name="absorb_step", kind="project", rows=64, heads=16, n_in=128, n_out=512, w_rows=True, handle=True),
        # a prompt's attention results out of the latent's columns
        dict(name="values_prompt", kind="project", rows=8192, heads=16, n_in=512, n_out=128, w_rows=False,
             handle=False),
        # keys and values of a question's tokens
        dict(name="expand_short", kind="expand", requests=4, keys=500, ragged=True, heads=16, latent=512, n_out=256,
             page=16, handle=False),
        # keys and values of a recalled context
        dict(name="expand_recall", kind="expand", requests=1, keys=16384, ragged=False, heads=16, latent=512,
             n_out=256, page=16, handle=False),
        # first tokens after one short cached chunk: latency
        _latent("latent_short", handle=True),
        # a batch of ragged requests, as a server decodes them
        _latent("latent_batch", requests=64, keys=8192, ragged=True, handle=True),
        # one request decodes over a long recall, a few speculated tokens at once
        _latent("latent_recall", keys=65536, queries=3, lse=True, handle=True),
        # wide rows: 128 heads read every latent
        _latent("latent_wide", requests=16, queries=2, keys=8192, ragged=True, heads=128, page=64),
        # a prompt chunk of 1024 tokens over a recalled context
        _expanded("expanded_chunk", queries=1024, keys=16384),
        # ragged prompts of eight requests, most of their keys their own
        _expanded("expanded_ragged", requests=8, queries=1024, ragged_q=True, keys=2048, ragged=True, page=64,
                  lse=True),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], even over its logarithm."""
    return int(min(hi, max(lo, round(float(lo) * (float(hi) / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["append", "append", "project", "project", "expand", "latent", "latent", "latent", "expanded",
                       "expanded"])
    page = rng.choice([16, 16, 32, 64])
    ragged = rng.random() < 0.7
    handle = rng.random() < 0.5
    heads = rng.choice([4, 8, 16, 16, 32, 128])
    if kind == "append":
        rows = rng.choice(["latent", "kv"])
        c = _append("", chunks=_log(rng, 1, 64), tokens=_log(rng, 1, 1024), before=rng.choice([0, _log(rng, 1, 8000)]),
                    ragged=ragged, page=page, rows=rows, pairing=rng.choice(["neox", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "turns", "pairs"]), handle=handle)
        del c["name"]
        if rows == "kv":
            c["heads"], group = rng.choice([(1, 8), (2, 6), (4, 7), (8, 8), (32, 1)])
            c["dim"] = rng.choice([64, 128])
            c["q_heads"] = c["heads"] * group
            c["rope_dim"] = rng.choice([c["dim"], c["dim"] // 2])
            c["sections"] = rng.random() < 0.3
        else:
            c["dim"] = rng.choice([576, 320])
            c["q_heads"] = heads
        while c["chunks"] * c["tokens"] * (2 * c["heads"] * c["dim"] + c["q_heads"] * c["rope_dim"]) > 3 << 25:
            c["tokens"] = max(1, c["tokens"] // 2)
        return c
    if kind == "project":
        n_in, n_out = rng.choice([(128, 512), (512, 128), (64, 256), (256, 64), (192, 320)])
        c = dict(kind=kind, rows=_log(rng, 1, 8192), heads=heads, n_in=n_in, n_out=n_out, w_rows=rng.random() < 0.5,
                 handle=handle)
        while c["rows"] * heads * (n_in + n_out) > 8192 * 16 * 640:
            c["rows"] //= 2
        return c
    if kind == "expand":
        latent, n_out = rng.choice([(512, 256), (512, 256), (256, 128), (512, 128)])
        c = dict(kind=kind, requests=_log(rng, 1, 32), keys=_log(rng, 1, 16384), ragged=ragged, heads=heads,
                 latent=latent, n_out=n_out, page=page, handle=handle)
        while c["requests"] * c["keys"] * heads * n_out * latent > 16384 * 4096 * 512:
            c["requests" if c["requests"] > 1 else "keys"] //= 2
        return c
    if kind == "latent":
        queries = 1 if rng.random() < 0.5 else _log(rng, 2, 64)
        c = _latent("", requests=_log(rng, 1, 64), queries=queries, ragged_q=rng.random() < 0.5,
                    keys=_log(rng, max(queries, 40), 65536), ragged=ragged, heads=heads,
                    latent=rng.choice([512, 512, 512, 256]), page=page, causal=rng.random() < 0.85,
                    lse=rng.random() < 0.3, handle=handle)
    else:
        queries = _log(rng, 2, 1024)
        c = _expanded("", requests=_log(rng, 1, 32), queries=queries, ragged_q=rng.random() < 0.5,
                      keys=_log(rng, max(queries, 40), 16384), ragged=ragged, heads=min(heads, 32),
                      dim=rng.choice([128, 128, 64]), page=page, causal=rng.random() < 0.85, lse=rng.random() < 0.3,
                      handle=handle)
    del c["name"]
    if c["causal"] and rng.random() < 0.25:
        c["window"] = _log(rng, 16, 4096)
    # no more than the largest listed ones read and compute (a window is not counted: plain forms make every product)
    whole = dict(c, window=0)
    while work(whole)["bytes"] > 350e6 or work(whole)["flops"] > 160e9:
        if c["requests"] > 1:
            c["requests"] = max(1, c["requests"] // 2)
        elif c["keys"] // 2 >= queries:
            c["keys"] //= 2
        else:
            c["heads"] //= 2
        whole = dict(c, window=0)
    return c


def _spread(n, lo, hi, ragged):
    """n lengths in [lo, hi]: all hi, or spread evenly over the range in a mixed order."""
    if not ragged or n == 1:
        return [hi] * n
    return [lo + int((hi - lo + 0.999) * ((0.5 + 0.6180339887498949 * i) % 1.0)) for i in range(n)]


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


def _starts(lengths):
    return [sum(lengths[:r]) for r in range(len(lengths))]


# the scaled positions of the cases: contexts of 8192 tokens stretched
SCALING = {"linear": dict(factor=4.0, amplitude=1.0), "turns": dict(factor=8.0, low=1.0, high=4.0, amplitude=1.0),
           "pairs": dict(factor=4.0, low=1.0, high=32.0, amplitude=1.125)}
ORIGINAL = 8192


def _theta(case):
    return 1e4 if case["rows"] == "latent" else 1e6


def _sections(case):
    """Pairs that turn by the time, height and width coordinates."""
    half = case["rope_dim"] // 2
    return (half - 2 * (half // 3), half // 3, half // 3)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(shape, gen, std=1.0):
    out = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 26):
        b = min(flat.numel(), a + (1 << 26))
        flat[a:b] = torch.randn(b - a, generator=gen, device=DEV) * std
    return out


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _tables(lengths, page, gen):
    """An injective page table [requests, pages] over a pool in random order (unused entries -1), and
    the number of pool pages (one in sixteen unused)."""
    need = [_pages(n, page) for n in lengths]
    total = max(1, sum(need))
    pool = total + total // 16 + 1
    order = torch.randperm(pool, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((len(lengths), max([1] + need)), -1, dtype=torch.int32, device=DEV)
    rows = torch.tensor([r for r, n in enumerate(need) for _ in range(n)], dtype=torch.long, device=DEV)
    cols = torch.tensor([j for n in need for j in range(n)], dtype=torch.long, device=DEV)
    table[rows, cols] = order[:sum(need)]
    return table, pool


def _whiten(cache, table, lengths, page):
    """NaN in the slots of a cache [pages, page, ...] that no token uses, as memory holds before its first use."""
    used = torch.zeros(cache.shape[0], page, dtype=torch.bool, device=DEV)
    n = torch.tensor(lengths, device=DEV)
    at = torch.arange(table.shape[1] * page, device=DEV).view(-1, page)
    ok = at[None] < n[:, None, None]
    pages = table.long().clamp(min=0)[:, :, None].expand_as(ok)
    inner = torch.arange(page, device=DEV).expand_as(ok)
    used[pages[ok], inner[ok]] = True
    cache[~used] = float("nan")


def prepare(case, seed):
    gen = _gen(seed)
    kind = case["kind"]
    s = {"case": case, "kept": {}}
    if kind == "append":
        before, tokens = _append_lengths(case)
        table, pool = _tables([b + t for b, t in zip(before, tokens)], case["page"], gen)
        n, H, D, page = sum(tokens), case["heads"], case["dim"], case["page"]
        if case["rows"] == "latent":
            s.update(k=_randn((1, n, 1, D), gen), v=None, kc=_randn((1, pool, page, 1, D), gen), vc=None)
            # the band of the queries' columns, turned into the absorbed queries' rows
            s["q"] = _randn((1, n, case["q_heads"], 128 + ROPE), gen)[..., 128:]
            s["q_out"] = _randn((1, n, case["q_heads"], D), gen)[..., D - ROPE:]
        else:
            rows, cache = _randn((1, n, 2, H, D), gen), _randn((1, pool, page, 2, H, D), gen)
            s.update(k=rows[:, :, 0], v=rows[:, :, 1], kc=cache[:, :, :, 0], vc=cache[:, :, :, 1])
            s["q"] = _randn((1, n, case["q_heads"], D), gen)[..., :case["rope_dim"]]
            s["q_out"] = _randn((1, n, case["q_heads"], D), gen)[..., :case["rope_dim"]]
        if case["sections"]:
            s["positions"] = torch.randint(0, 32768, (n, 3), generator=gen, device=DEV, dtype=torch.int32)
        s.update(table=table, before=_i32(before), tokens=_i32(tokens), base=_i32(_starts(tokens)), n=max(tokens))
        return s
    if kind == "project":
        H, a, b = case["heads"], case["n_in"], case["n_out"]
        s["x"] = _randn((case["rows"], H, a), gen)
        w = _randn((H, a, b) if case["w_rows"] else (H, b, a), gen, a ** -0.5)
        s["w"] = w if case["w_rows"] else w.transpose(1, 2)
        s["out"] = torch.zeros((case["rows"], H, b), dtype=torch.bfloat16, device=DEV)
        return s
    lengths, H, page = _key_lengths(case), case["heads"], case["page"]
    table, pool = _tables(lengths, page, gen)
    latent = case.get("latent", 512)
    cache = _randn((pool, page, latent + ROPE), gen)
    _whiten(cache, table, lengths, page)
    s.update(cache=cache, table=table, kv=_i32(lengths), n_keys=max(lengths), kv_base=_i32(_starts(lengths)))
    if kind == "expand":
        n = case["n_out"]
        s["w"] = _randn((H, n, latent), gen, latent ** -0.5).transpose(1, 2)
        s["out"] = torch.zeros((sum(lengths), H, n), dtype=torch.bfloat16, device=DEV)
        return s
    nq = _query_lengths(case)
    s.update(nq=_i32(nq), base=_i32(_starts(nq)), n_queries=max(nq))
    if kind == "latent":
        # queries absorbed into the latent: of the size that a head's 128 columns give
        s["q"] = _randn((sum(nq), H, latent + ROPE), gen, 0.5)
        s["out"] = torch.zeros((sum(nq), H, latent), dtype=torch.bfloat16, device=DEV)
        s["scale"] = (128 + ROPE) ** -0.5
    else:
        D = case["dim"]
        rows = _randn((sum(lengths), H, 2 * D), gen)
        s.update(k=rows[..., :D], v=rows[..., D:])
        s["q"] = _randn((sum(nq), H, D + ROPE), gen)
        s["out"] = torch.zeros((sum(nq), H, D), dtype=torch.bfloat16, device=DEV)
        s["scale"] = (D + ROPE) ** -0.5
    if case["lse"]:
        s["lse"] = torch.zeros((sum(nq), H), device=DEV)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return _OWN[state["case"]["kind"]](state) if own else _PLAIN[state["case"]["kind"]](state)


def _call(s, prepare_call, direct_call, *a, **kw):
    """A program with fixed buffers prepares a call once and launches it each step; one whose tensors
    change makes the whole call."""
    if not s["case"]["handle"]:
        return direct_call(*a, **kw)
    if "call" not in s["kept"]:
        s["kept"]["call"] = prepare_call(*a, **kw)
    s["kept"]["call"].launch()


def _own_append(s):
    km, c = _km(), s["case"]
    latent = c["rows"] == "latent"
    rope = km.RopeSpec(theta=_theta(c), rope_dim=c["rope_dim"], rope_offset=c["dim"] - ROPE if latent else 0,
                       pairing=c["pairing"], sections=_sections(c) if c["sections"] else None)
    scaling = None
    if c["scaling"] != "none":
        f = SCALING[c["scaling"]]
        scaling = km.RopeScaling(kind=c["scaling"], factor=f["factor"], original_tokens=ORIGINAL,
                                 low_turns=f.get("low", 1.0), high_turns=f.get("high", 32.0),
                                 amplitude=f["amplitude"])
    _call(s, km.prepare_append_rotated, km.append_rotated, s["k"], s["v"], s["kc"], s["vc"], s["table"], rope=rope,
          scaling=scaling, positions=s.get("positions"), n_tokens=s["n"], tokens_before=s["before"],
          chunk_tokens=s["tokens"], row_base=s["base"], q=s["q"], q_out=s["q_out"])
    return _append_result(s, s["kc"], s["vc"], s["q_out"])


def _append_result(s, k, v, q):
    return {"k": k, "q": q} if v is None else {"k": k, "v": v, "q": q}


def _own_project(s):
    km = _km()
    _call(s, km.prepare_project_heads, km.project_heads, s["x"], s["w"], s["out"])
    return {"out": s["out"]}


def _own_expand(s):
    km = _km()
    _call(s, km.prepare_expand_latent, km.expand_latent, s["cache"], s["w"], s["out"], s["table"], s["kv"],
          n_keys=s["n_keys"], row_base=s["kv_base"])
    return {"out": s["out"]}


def _attend_kw(s):
    c = s["case"]
    return dict(n_queries=s["n_queries"], n_keys=s["n_keys"], q_base=s["base"], q_tokens=s["nq"], scale=s["scale"],
                causal=c["causal"], window=c["window"], lse=s.get("lse"))


def _own_latent(s):
    km = _km()
    _call(s, km.prepare_attend_latent, km.attend_latent, s["q"], s["cache"], s["out"], s["table"], s["kv"],
          **_attend_kw(s))
    return {"out": s["out"], "lse": s["lse"]} if s["case"]["lse"] else {"out": s["out"]}


def _own_expanded(s):
    km = _km()
    _call(s, km.prepare_attend_expanded, km.attend_expanded, s["q"], s["k"], s["v"], s["cache"][..., -ROPE:],
          s["out"], s["table"], s["kv"], kv_base=s["kv_base"], **_attend_kw(s))
    return {"out": s["out"], "lse": s["lse"]} if s["case"]["lse"] else {"out": s["out"]}


_OWN = {"append": _own_append, "project": _own_project, "expand": _own_expand, "latent": _own_latent,
        "expanded": _own_expanded}


# ---------------------------------------------------------------------------
# plain forms, 32 bits (angles in 64)
# ---------------------------------------------------------------------------

def _frequencies(case):
    """Radians a position of every pair, and the factor on both rotated columns."""
    half = case["rope_dim"] // 2
    j = torch.arange(half, dtype=torch.float64, device=DEV)
    theta = _theta(case)
    freq = torch.exp(-math.log(theta) * 2 * j / case["rope_dim"])
    kind = case["scaling"]
    if kind == "none":
        return freq, 1.0
    f = SCALING[kind]
    if kind == "linear":
        return freq / f["factor"], f["amplitude"]
    if kind == "turns":
        # the share that keeps its frequency grows with the turns a pair makes over the original context
        keep = (ORIGINAL * freq / (2 * math.pi) - f["low"]) / (f["high"] - f["low"])
    else:
        # ... or with the pair's number, between those that make `high` and `low` turns
        at = [half * math.log(ORIGINAL / (2 * math.pi * t)) / math.log(theta) for t in (f["high"], f["low"])]
        first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), case["rope_dim"] - 1)
        keep = 1 - (j - first) / max(last - first, 0.001)
    keep = keep.clamp(0, 1)
    return freq * (keep + (1 - keep) / f["factor"]), f["amplitude"]


def _angles(s):
    """Radians [rows, pairs] of every packed row, 64 bits."""
    c = s["case"]
    freq, amplitude = _frequencies(c)
    if c["sections"]:
        coord = torch.tensor([i for i, n in enumerate(_sections(c)) for _ in range(n)], device=DEV)
        return s["positions"][:, coord].double() * freq, amplitude
    r = torch.repeat_interleave(torch.arange(c["chunks"], device=DEV), s["tokens"].long())
    at = torch.arange(r.numel(), device=DEV) - s["base"].long()[r] + s["before"].long()[r]
    return at.double()[:, None] * freq, amplitude


def _turned(x, cos, sin, pairing):
    """x [..., pairs * 2] with its pairs turned by cos, sin [rows, 1, pairs]."""
    if pairing == "neox":
        a, b = x.chunk(2, dim=-1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)


def _plain_append(s):
    c = s["case"]
    angle, amplitude = _angles(s)
    cos, sin = (torch.cos(angle) * amplitude).float()[:, None], (torch.sin(angle) * amplitude).float()[:, None]
    r = torch.repeat_interleave(torch.arange(c["chunks"], device=DEV), s["tokens"].long())
    tok = torch.arange(r.numel(), device=DEV) - s["base"].long()[r] + s["before"].long()[r]
    page, inner = s["table"][r, tok // c["page"]].long(), tok % c["page"]
    o = c["dim"] - ROPE if c["rows"] == "latent" else 0
    k = s["k"][0].float()
    band = _turned(k[..., o:o + c["rope_dim"]], cos, sin, c["pairing"])
    k = torch.cat([k[..., :o], band, k[..., o + c["rope_dim"]:]], dim=-1)
    s["kc"][0, page, inner] = k.to(torch.bfloat16)
    if s["v"] is not None:
        s["vc"][0, page, inner] = s["v"][0]
    s["q_out"].copy_(_turned(s["q"].float(), cos, sin, c["pairing"]).to(torch.bfloat16))
    return _append_result(s, s["kc"], s["vc"], s["q_out"])


def _plain_project(s):
    x, w = s["x"].float().transpose(0, 1).contiguous(), s["w"].float().contiguous()
    return {"out": torch.matmul(x, w).transpose(0, 1).to(torch.bfloat16).contiguous()}


def _gathered(s):
    """The pool's rows of every request, packed [rows, columns]."""
    c = s["case"]
    r = torch.repeat_interleave(torch.arange(c["requests"], device=DEV), s["kv"].long())
    tok = torch.arange(r.numel(), device=DEV) - s["kv_base"].long()[r]
    return s["cache"][s["table"][r, tok // c["page"]].long(), tok % c["page"]]


def _plain_expand(s):
    c = s["case"]
    x = _gathered(s)[:, :c["latent"]].float()
    w = s["w"].float().permute(1, 0, 2).reshape(c["latent"], -1)
    return {"out": torch.matmul(x, w).view(-1, c["heads"], c["n_out"]).to(torch.bfloat16)}


def _padded(s, rows, base, lengths, most):
    """Packed rows [n, ...] as [requests, most, ...] in 32 bits, zero past a request's length."""
    i = torch.arange(most, device=DEV)
    at = (base.long()[:, None] + i).clamp(max=rows.shape[0] - 1)
    there = i[None] < lengths.long()[:, None]
    x = rows[at].float()
    return torch.where(there.view(*there.shape, *([1] * (x.dim() - 2))), x, 0.0)


def _plain_attend(s, q, k, v):
    """q [R, nq, H, D], k and v [R, H or 1, n, D]; the packed results."""
    c = s["case"]
    R, nq, H, D = q.shape
    kv, n = s["kv"].long(), k.shape[2]
    nqs = s["nq"].long()
    pos, i = torch.arange(n, device=DEV), torch.arange(nq, device=DEV)
    if k.shape[1] == 1:
        q = q.reshape(R, 1, nq * H, D)
    else:
        q = q.transpose(1, 2).contiguous()
    sc = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    last = (kv - nqs)[:, None] + i if c["causal"] else (kv - 1)[:, None].expand(R, nq)
    seen = (pos < kv[:, None, None]) & (pos <= last[..., None])
    if c["window"]:
        seen = seen & (pos > last[..., None] - c["window"])
    if k.shape[1] == 1:
        seen = seen[:, :, None].expand(R, nq, H, n).reshape(R, 1, nq * H, n)
    else:
        seen = seen[:, None]
    sc = sc.masked_fill_(~seen, float("-inf"))
    m = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - torch.where(torch.isfinite(m), m, 0.0))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    lse = (torch.log(total) + m).squeeze(-1)
    if k.shape[1] == 1:
        o, lse = o.view(R, nq, H, -1), lse.view(R, nq, H)
    else:
        o, lse = o.transpose(1, 2), lse.transpose(1, 2)
    real = i[None] < nqs[:, None]
    got = {"out": o[real].to(torch.bfloat16)}
    if c["lse"]:
        got["lse"] = lse[real]
    return got


def _plain_latent(s):
    c = s["case"]
    rows = _padded(s, _gathered(s), s["kv_base"], s["kv"], s["n_keys"])[:, None]
    q = _padded(s, s["q"], s["base"], s["nq"], s["n_queries"])
    return _plain_attend(s, q, rows, rows[..., :c["latent"]].contiguous())


def _plain_expanded(s):
    D, H = s["case"]["dim"], s["case"]["heads"]
    k = _padded(s, s["k"], s["kv_base"], s["kv"], s["n_keys"]).transpose(1, 2)
    v = _padded(s, s["v"], s["kv_base"], s["kv"], s["n_keys"]).transpose(1, 2).contiguous()
    rope = _padded(s, _gathered(s)[:, -ROPE:], s["kv_base"], s["kv"], s["n_keys"])[:, None].expand(-1, H, -1, -1)
    q = _padded(s, s["q"], s["base"], s["nq"], s["n_queries"])
    return _plain_attend(s, q, torch.cat([k, rope], dim=-1), v)


_PLAIN = {"append": _plain_append, "project": _plain_project, "expand": _plain_expand, "latent": _plain_latent,
          "expanded": _plain_expanded}


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
    kind, H = case["kind"], case["heads"]
    if kind == "append":
        before, tokens = _append_lengths(case)
        n = sum(tokens)
        row = case["dim"] if case["rows"] == "latent" else 2 * H * case["dim"]
        got = 4.0 * n * (row + case["q_heads"] * case["rope_dim"])
        got += 4.0 * sum(_pages(b + t, case["page"]) - b // case["page"] for b, t in zip(before, tokens))
        if case["sections"]:
            got += 12.0 * n
        return {"bytes": got, "flops": 3.0 * n * case["rope_dim"] * (H + case["q_heads"])}
    if kind == "project":
        n, a, b = case["rows"], case["n_in"], case["n_out"]
        return {"bytes": 2.0 * H * (n * (a + b) + a * b), "flops": 2.0 * n * H * a * b}
    lengths = _key_lengths(case)
    if kind == "expand":
        n, a, b = sum(lengths), case["latent"], case["n_out"]
        return {"bytes": 2.0 * (n * (a + H * b) + H * a * b) + 4.0 * n / case["page"], "flops": 2.0 * n * H * a * b}
    nq = _query_lengths(case)
    keys = pairs = 0
    for n, m in zip(lengths, nq):
        a, b = _visible(case, n, m)
        keys, pairs = keys + a, pairs + b
    if kind == "latent":
        d, dv, row = case["latent"] + ROPE, case["latent"], case["latent"] + ROPE
    else:
        d, dv, row = case["dim"] + ROPE, case["dim"], 2 * H * case["dim"] + ROPE
    got = 2.0 * row * keys + 2.0 * sum(nq) * H * (d + dv) + 4.0 * keys / case["page"]
    if case["lse"]:
        got += 4.0 * sum(nq) * H
    return {"bytes": got, "flops": 2.0 * H * (d + dv) * pairs}


# ---------------------------------------------------------------------------
# the definition, 64 bits
# ---------------------------------------------------------------------------

def _rows64(s, r, n):
    """The first n rows of request r in the pool."""
    page = s["case"]["page"]
    return s["cache"][s["table"][r, :_pages(n, page)].long()].flatten(0, 1)[:n].double()


def _attend64(q, k, v, scale, low, top):
    """Rows q [m, D] over keys [low[i], top[i]) of k, v."""
    z = torch.matmul(q, k.t().contiguous()) * scale
    j = torch.arange(k.shape[0], device=DEV)
    z.masked_fill_((j[None] >= top[:, None]) | (j[None] < low[:, None]), -math.inf)
    lse = torch.logsumexp(z, -1)
    w = torch.exp(z - torch.where(torch.isinf(lse), 0.0, lse)[:, None])
    return torch.matmul(w, v), lse


def exact(case, seed):
    kind, H = case["kind"], case["heads"]
    s = prepare(case, seed)
    if kind == "append":
        return _exact_append(case, s)
    if kind == "project":
        out = torch.empty(s["out"].shape, dtype=torch.float64, device=DEV)
        for h in range(H):
            out[:, h] = torch.matmul(s["x"][:, h].double(), s["w"][h].double())
        return {"out": out}
    lengths = _key_lengths(case)
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    if kind == "expand":
        at = 0
        for r, n in enumerate(lengths):
            x = _rows64(s, r, n)[:, :case["latent"]]
            for h in range(H):
                out[at:at + n, h] = torch.matmul(x, s["w"][h].double())
            at += n
        return {"out": out}
    nq, at, key = _query_lengths(case), 0, 0
    if sum(n * m for n, m in zip(lengths, nq)) * H > 2 << 30:
        return None
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device=DEV)
    for r, (n, m) in enumerate(zip(lengths, nq)):
        i = torch.arange(m, device=DEV)
        top = (n - m + 1 + i) if case["causal"] else torch.full_like(i, n)
        low = (top - case["window"]).clamp(min=0) if case["window"] else torch.zeros_like(top)
        pool = _rows64(s, r, n)
        if kind == "latent":
            q = s["q"][at:at + m].double().flatten(0, 1)
            o, z = _attend64(q, pool, pool[:, :case["latent"]], s["scale"], low.repeat_interleave(H),
                             top.repeat_interleave(H))
            out[at:at + m], lse[at:at + m] = o.view(m, H, -1), z.view(m, H)
        else:
            for h in range(H):
                k = torch.cat([s["k"][key:key + n, h].double(), pool[:, -ROPE:]], dim=1)
                out[at:at + m, h], lse[at:at + m, h] = _attend64(s["q"][at:at + m, h].double(), k,
                                                                 s["v"][key:key + n, h].double(), s["scale"], low, top)
        at, key = at + m, key + n
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def _exact_append(case, s):
    """Row by row in complex numbers: a pair (x, y) becomes (x + i y) e^(i angle)."""
    before, tokens = _append_lengths(case)
    half, theta = case["rope_dim"] // 2, _theta(case)
    sections = _sections(case)
    freq, amplitude, coord = [], 1.0, []
    for j in range(half):
        w = theta ** (-j / half)
        f = SCALING.get(case["scaling"])
        if f is not None:
            amplitude = f["amplitude"]
            share = 0.0                                    # of the unscaled frequency
            if case["scaling"] == "turns":
                share = (ORIGINAL * w / (2 * math.pi) - f["low"]) / (f["high"] - f["low"])
            elif case["scaling"] == "pairs":
                def pair(turns):
                    return half * math.log(ORIGINAL / (turns * 2 * math.pi)) / math.log(theta)
                lo, hi = max(0, math.floor(pair(f["high"]))), min(2 * half - 1, math.ceil(pair(f["low"])))
                share = 1 - (j - lo) / (hi - lo if hi > lo else 0.001)
            share = min(1.0, max(0.0, share))
            w = w / f["factor"] + share * (w - w / f["factor"])
        freq.append(w)
        coord.append(0 if j < sections[0] else 1 if j < sections[0] + sections[1] else 2)
    freq = torch.tensor(freq, dtype=torch.float64, device=DEV)

    def turn(x, at):
        z = torch.complex(x[..., :half], x[..., half:]) if case["pairing"] == "neox" else \
            torch.view_as_complex(x.unflatten(-1, (half, 2)).contiguous())
        z = z * (amplitude * torch.polar(torch.ones_like(at), at))[:, None]
        return torch.cat([z.real, z.imag], -1) if case["pairing"] == "neox" else torch.view_as_real(z).flatten(-2)

    o = case["dim"] - ROPE if case["rows"] == "latent" else 0
    k, q = s["kc"].double(), torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    v = None if s["v"] is None else s["vc"].double()
    first = 0
    for c, (b, t) in enumerate(zip(before, tokens)):
        rows = slice(first, first + t)
        if case["sections"]:
            at = s["positions"][rows].double()[:, coord] * freq
        else:
            at = torch.arange(b, b + t, dtype=torch.float64, device=DEV)[:, None] * freq
        q[0, rows] = turn(s["q"][0, rows].double(), at)
        x = s["k"][0, rows].double()
        x[..., o:o + 2 * half] = turn(x[..., o:o + 2 * half].clone(), at)
        tok = torch.arange(b, b + t, device=DEV)
        pg = s["table"][c].long()[tok // case["page"]]
        k[0, pg, tok % case["page"]] = x
        if v is not None:
            v[0, pg, tok % case["page"]] = s["v"][0, rows].double()
        first += t
    return _append_result(s, k, v, q)
