"""Plain 64-bit forms of the paged-cache operators for the tests, from their
definitions in include/kamera.h.  numpy only; e4m3 is decoded and rounded here
by its definition (4 exponent bits, bias 7, 3 fraction bits, largest value 448,
0x7f / 0xff NaN)."""

from __future__ import annotations

import math

import numpy as np

TOP8 = 448.0
MIN_EXP = -100


def e4m3_values() -> np.ndarray:
    """The 256 values, in 64 bits."""
    v = np.empty(256)
    for b in range(256):
        s, e, f = -1.0 if b & 0x80 else 1.0, (b >> 3) & 15, b & 7
        v[b] = s * (f / 8.0 * 2.0 ** -6 if e == 0 else (1 + f / 8.0) * 2.0 ** (e - 7))
        if b & 0x7F == 0x7F:
            v[b] = math.nan
    return v


_VALUES = e4m3_values()
_POS = _VALUES[:127]                      # 0 .. 448, ascending


def decode(b: np.ndarray) -> np.ndarray:
    return _VALUES[b]


def encode(x: np.ndarray) -> np.ndarray:
    """The nearest e4m3 byte, ties to the even byte; what is not finite gives NaN (0x7f)."""
    a = np.abs(x)
    with np.errstate(invalid="ignore"):
        hi = np.clip(np.searchsorted(_POS, a, side="left"), 1, 126)
        lo = hi - 1
        dl, dh = a - _POS[lo], _POS[hi] - a
        pick = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    pick = np.where(a == 0, 0, pick)
    b = (pick | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)
    return np.where(np.isfinite(x), b, 0x7F).astype(np.uint8)


def least_exp(amax: float, top: float) -> int:
    """The least e >= MIN_EXP with amax <= top * 2^e."""
    if amax == 0:
        return MIN_EXP
    e = math.frexp(amax / top)[1] - 1
    while amax > math.ldexp(top, e):
        e += 1
    while amax <= math.ldexp(top, e - 1):
        e -= 1
    return max(e, MIN_EXP)


def finite_max(x: np.ndarray) -> float:
    a = np.abs(x[np.isfinite(x)])
    return float(a.max()) if a.size else 0.0


def page_tables(before, after, free, begin, table, page, pool, n_slots):
    """(table, base, slots, end, flags) after one call; flags a set of texts."""
    table, flags = table.copy(), set()
    cap = table.shape[1] * page
    base, slots, at = [0], [], begin
    for r, a in enumerate(after):
        a = max(int(a), 0)
        if a > cap:
            flags.add("length")
            a = cap
        b = min(max(int(before[r]), 0) if before is not None else 0, a)
        for j in range(-(-b // page), -(-a // page)):
            pg = -1
            if at >= len(free):
                flags.add("none")
            elif not 0 <= free[at] < pool:
                flags.add("page")
            else:
                pg = int(free[at])
            table[r, j] = pg
            at += 1
        for t in range(b, a):
            pg = int(table[r, t // page])
            if not 0 <= pg < pool:
                if pg != -1 or t // page < -(-b // page):
                    flags.add("page")
                pg = -1
            slots.append(pg * page + t % page if pg >= 0 else -1)
        base.append(len(slots))
    slots = (slots + [-1] * n_slots)[:n_slots]
    return table, np.array(base), np.array(slots), min(at, len(free)), flags


def append(rows, cache, scale, table, before, tokens, page, sums=None):
    """One layer and plane: rows[c] [tokens, H, D] into cache [pages, page, H, D] (bytes) and scale [pages, H],
    in place; sums: (k_sum [pages, H, D], k_sum_scale [pages, H])."""
    for c, (b, n) in enumerate(zip(before, tokens)):
        for j in range(b // page, -(-(b + n) // page)):
            pg = int(table[c, j])
            if not 0 <= pg < cache.shape[0]:
                continue
            lo, hi = max(b - j * page, 0), min(b + n - j * page, page)
            if hi <= lo:
                continue
            for h in range(cache.shape[2]):
                x = rows[c][j * page + lo - b:j * page + hi - b, h]
                e = least_exp(finite_max(x), TOP8)
                if lo > 0:
                    e_old = int(round(math.log2(scale[pg, h])))
                    if e > e_old:
                        cache[pg, :lo, h] = encode(np.ldexp(decode(cache[pg, :lo, h]), e_old - e))
                    e = max(e, e_old)
                cache[pg, lo:hi, h] = encode(np.ldexp(x, -e))
                scale[pg, h] = 2.0 ** e
                if sums is not None and hi == page:
                    t = np.nan_to_num(decode(cache[pg, :, h])).sum(0)
                    f = least_exp(finite_max(t), 127.0)
                    sums[0][pg, h] = np.rint(np.ldexp(t, -f)).astype(np.int8)
                    sums[1][pg, h] = np.float32(math.ldexp(1.0, e + f))     # 0 where fp32 has no such power


def select(q, k_sum, k_sum_scale, table, kv, page, keep, first, last):
    """[list of page indices] for each (request, head)."""
    R, HQ, _ = q.shape
    H = k_sum.shape[1]
    G = HQ // H
    got = []
    for r in range(R):
        n = -(-int(kv[r]) // page)
        for h in range(H):
            if n <= keep:
                got.append(list(range(n)))
                continue
            x = np.where(np.isfinite(q[r, h * G:(h + 1) * G]), q[r, h * G:(h + 1) * G], 0.0)
            f = least_exp(float(np.abs(x).max()), 127.0)
            q8 = np.rint(np.ldexp(x, -f))
            s = []
            for j in range(n):
                pg = int(table[r, j])
                ok = 0 <= pg < k_sum.shape[0]
                v = float((q8 @ k_sum[pg, h].astype(float)).max()) * float(k_sum_scale[pg, h]) if ok else -math.inf
                s.append(math.inf if j < first or j >= n - last else v)
            order = sorted(range(n), key=lambda j: (-s[j], j))[:keep]
            got.append(sorted(order))
    return got


def attend_row(q, k, v, seen, scale):
    """(out, lse) of one query row over the keys with seen[t], 64 bits."""
    if not seen.any():
        return np.zeros(v.shape[1]), -math.inf
    s = (k[seen] @ q) * scale
    with np.errstate(invalid="ignore"):
        m = s.max()
        p = np.exp(s - m)
        return p @ v[seen] / p.sum(), m + math.log(p.sum()) if np.isfinite(m) else math.nan


def attend(q, k, v, table, kv, nq, base, page, scale, causal=True, window=0, sel=None):
    """q [rows, HQ, D]; k, v [pages, page, H, D] as values; sel: per (request, head) lists of page indices.
    (out, lse) with NaN where no request has the row."""
    HQ, H = q.shape[1], k.shape[2]
    G = HQ // H
    out, lse = np.full(q.shape, math.nan), np.full(q.shape[:2], math.nan)
    for r in range(len(kv)):
        n = int(kv[r])
        for h in range(H):
            pages = range(-(-n // page)) if sel is None else sel[r * H + h]
            pos = np.array([j * page + t for j in pages for t in range(page)], dtype=int)
            pg = np.array([int(table[r, j]) for j in pages for _ in range(page)], dtype=int)
            ok = (pos < n) & (pg >= 0) & (pg < k.shape[0])
            at = np.where(ok, pg, 0)
            kk, vv = k[at, pos % page, h], v[at, pos % page, h]
            for i in range(nq[r]):
                last = n - nq[r] + i if causal else n - 1
                seen = ok & (pos <= last)
                if window:
                    seen &= pos > last - window
                for g in range(h * G, (h + 1) * G):
                    out[base[r] + i, g], lse[base[r] + i, g] = attend_row(q[base[r] + i, g], kk, vv, seen, scale)
    return out, lse
