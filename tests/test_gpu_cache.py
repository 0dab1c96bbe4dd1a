"""The paged-cache operators on the GPU against plain 64-bit forms (cache_ref).

Bounds.  Whole numbers, cache bytes and scales are equal.  For attention, with
A = sum_t p_t |V_t| of an output element (64 bits):
  p is rounded to bf16 (8 significant bits) before the product with V   <= 2^-8 A
  the output is rounded to bf16                                         <= 2^-8 |out| <= 2^-8 A
  scores, exponentials and sums in fp32                                 <= 2^-11 A for the scores here
so |out - ref| <= (2^-7 + 2^-11) A.  A score is a sum of D <= 128 fp32 products
with sum |q_j k_j| * scale <= 32 in these inputs: off by at most 128 * 2^-24 * 32
< 2^-11, which bounds p's relative error and the error of lse.
"""

from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2606_23581_amd as km
from tests import cache_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"
BOUND = 2.0 ** -7 + 2.0 ** -11


def i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device=DEV)


def bf16(x):
    """float64 numpy -> (bf16 device tensor, its values)."""
    t = torch.tensor(np.asarray(x, dtype=np.float32)).to(torch.bfloat16)
    return t.to(DEV), t.double().numpy()


def table_for(rng, lengths, page, width=None, spare=3):
    need = [-(-n // page) for n in lengths]
    pool = sum(need) + spare
    order = rng.permutation(pool)
    width = max([1, width or 0] + need)
    t = np.full((len(lengths), width), -1, dtype=np.int32)
    at = 0
    for r, n in enumerate(need):
        t[r, :n] = order[at:at + n]
        at += n
    return t, pool


# ---------------------------------------------------------------------------
# page tables
# ---------------------------------------------------------------------------

TABLE_CASES = {
    "one_token": dict(before=[5], after=[6], page=16),
    "first_tokens": dict(before=None, after=[1, 16, 17, 0, 33], page=16),
    "steps": dict(before=[15, 16, 17, 31, 32, 0], after=[16, 17, 18, 32, 33, 1], page=16),
    "shrink_negative": dict(before=[20, -3, 7], after=[4, 9, -1], page=8),
    "odd_page": dict(before=[0, 10, 3], after=[50, 11, 40], page=7),
    "page_of_one": dict(before=[2, 0], after=[5, 4], page=1),
    "short_list": dict(before=[0, 0, 0], after=[40, 40, 40], page=16, n_free=5),
    "no_list": dict(before=[16, 3], after=[17, 5], page=16, n_free=0),
    "begin": dict(before=[0, 5], after=[30, 40], page=16, begin=4),
    "begin_past_end": dict(before=[0], after=[30], page=16, begin=99, n_free=10),
    "bad_free_page": dict(before=[0, 0], after=[60, 60], page=16, bad_free=2),
    "bad_old_page": dict(before=[20, 20], after=[30, 60], page=16, bad_old=True),
    "outgrow": dict(before=[10, 0, 30], after=[500, 20, 64], page=16, width=4),
    "few_slots": dict(before=[0, 0], after=[20, 20], page=16, n_slots=13),
    "no_slots": dict(before=[0, 0], after=[20, 20], page=16, n_slots=0),
    "many": dict(before=list(range(0, 700)), after=[b + (b * 7) % 40 for b in range(700)], page=16),
    "most": dict(before=None, after=[(r * 13) % 5 for r in range(8192)], page=2),
    "none": dict(before=None, after=[], page=16, n_slots=5),
}


@pytest.mark.parametrize("name", sorted(TABLE_CASES))
def test_page_tables(name):
    c = TABLE_CASES[name]
    rng = np.random.default_rng(3)
    before, after, page = c["before"], c["after"], c["page"]
    held = before if before is not None else [0] * len(after)
    width = c.get("width", max([1] + [-(-max(a, b, 0) // page) for a, b in zip(after, held)]) + 1)
    table, pool = table_for(rng, [min(max(b, 0), width * page) for b in held], page, width=width, spare=5)
    if c.get("bad_old"):
        table[0, 1] = -1
        table[1, 0] = pool + 7
    grow = sum(max(0, -(-max(a, 0) // page) - -(-max(b, 0) // page)) for a, b in zip(after, held))
    begin = c.get("begin", 0)
    n_free = c.get("n_free", grow + begin + 2)
    pool += n_free
    free = rng.permutation(np.arange(pool - n_free, pool)).astype(np.int32)
    if "bad_free" in c:
        free[c["bad_free"]] = pool
        free[c["bad_free"] + 1] = -5
    tokens = sum(max(0, max(a, 0) - max(b, 0)) for a, b in zip(after, held))
    n_slots = c.get("n_slots", tokens + 9)
    want = ref.page_tables(before, after, free, min(begin, n_free), table, page, pool, n_slots)
    t = i32(table.reshape(len(after), width))
    end, base, status = i32([-7]), i32(np.full(len(after) + 1, -7)), i32([0])
    slots = torch.full((n_slots,), -7, dtype=torch.int64, device=DEV) if "n_slots" not in c or n_slots else None
    km.page_tables(None if before is None else i32(before), i32(after), i32(free), t, page_size=page,
                   n_pool_pages=pool, free_begin=i32([begin]) if begin else None, free_end=end, token_base=base,
                   slots=slots, status=status)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(t.cpu().numpy(), want[0])
    np.testing.assert_array_equal(base.cpu().numpy(), want[1])
    if slots is not None:
        np.testing.assert_array_equal(slots.cpu().numpy(), want[2])
    assert int(end) == want[3]
    flags = (km.STATUS_NO_PAGE * ("none" in want[4]) | km.STATUS_BAD_LENGTH * ("length" in want[4])
             | km.STATUS_BAD_PAGE * ("page" in want[4] and slots is not None))
    assert int(status) == flags


# ---------------------------------------------------------------------------
# 8-bit append
# ---------------------------------------------------------------------------

def new_cache(rng, L, pool, page, H, D, layout):
    """Random bytes (NaN among them) and scales, as device views and as numpy."""
    b = rng.integers(0, 256, size=(L, pool, page, H, D), dtype=np.uint8)
    if layout == "heads":
        t = torch.tensor(b).to(DEV).transpose(2, 3).contiguous().transpose(2, 3)
    elif layout == "slots":                      # row order, wider rows than needed
        w = torch.zeros((L, pool, page, H + 1, D), dtype=torch.uint8, device=DEV)
        w[:, :, :, :H] = torch.tensor(b).to(DEV)
        t = w[:, :, :, :H]
    else:
        t = torch.tensor(b).to(DEV)
    e = rng.integers(-6, 3, size=(L, pool, H))
    return t, b.copy(), torch.tensor(2.0 ** e, dtype=torch.float32, device=DEV), 2.0 ** e


APPEND_CASES = {
    "fresh": dict(before=[0, 0], tokens=[16, 33], page=16),
    "single_tokens": dict(before=[0, 1, 15, 16, 17, 63], tokens=[1, 1, 1, 1, 1, 1], page=16),
    "odd": dict(before=[5, 31, 32, 0], tokens=[27, 1, 0, 70], page=32, H=3),
    "page64": dict(before=[10, 64, 63], tokens=[120, 64, 1], page=64, H=1),
    "d64": dict(before=[3, 0], tokens=[40, 16], page=16, D=64, H=5),
    "d64_page64": dict(before=[60, 1], tokens=[9, 63], page=64, D=64),
    "packed": dict(before=[0, 7, 20], tokens=[19, 25, 1], page=16, packed=True, L=2),
    "layers_slots": dict(before=[4, 0], tokens=[20, 20], page=16, L=3, layout="slots"),
    "zero_rows": dict(before=[0, 3], tokens=[16, 13], page=16, values="zero"),
    "huge": dict(before=[0, 3], tokens=[20, 13], page=16, values="huge"),
    "tiny": dict(before=[0, 3], tokens=[20, 13], page=16, values="tiny"),
    "lift": dict(before=[6, 15, 20], tokens=[10, 3, 5], page=16, values="lift"),
    "lift_far": dict(before=[6, 15, 20], tokens=[10, 3, 5], page=16, values="lift_far"),
    "nonfinite": dict(before=[0, 5, 9], tokens=[17, 11, 7], page=16, values="nonfinite"),
    "nonfinite_only": dict(before=[0], tokens=[16], page=16, values="nan"),
    "bad_page": dict(before=[0, 20], tokens=[20, 20], page=16, bad=True),
    "past_table": dict(before=[20], tokens=[20], page=16, cut=True),
}


@pytest.mark.parametrize("name", sorted(APPEND_CASES))
def test_append(name):
    c = APPEND_CASES[name]
    rng = np.random.default_rng(7)
    before, tokens, page = c["before"], c["tokens"], c["page"]
    L, H, D, C = c.get("L", 1), c.get("H", 2), c.get("D", 128), len(before)
    table, pool = table_for(rng, [b + t for b, t in zip(before, tokens)], page)
    if c.get("bad"):
        table[0, 1] = -1
        table[1, 1] = pool
    if c.get("cut"):
        table = table[:, :2].copy()
    n = max(tokens)
    x = rng.standard_normal((2, C, L, n, H, D)) * 2.0 ** rng.integers(-4, 4, size=(2, C, L, n, H, 1))
    v = c.get("values")
    if v == "zero":
        x[:] = 0
    elif v == "huge":
        x *= 2.0 ** 120
    elif v == "tiny":
        x *= 2.0 ** -122
    elif v in ("lift", "lift_far"):
        x *= 2.0 ** (9 if v == "lift" else 100)
    elif v == "nan":
        x[:] = np.nan
    elif v == "nonfinite":
        for a in (np.nan, np.inf, -np.inf):
            x[rng.random(x.shape) < 0.02] = a
    xt, xv = bf16(x)
    status = i32([0])
    kc, kb, ks, ksv = new_cache(rng, L, pool, page, H, D, c.get("layout", "heads"))
    vc, vb, vs, vsv = new_cache(rng, L, pool, page, H, D, c.get("layout", "dense"))
    sums = torch.full((L, pool, H, D), 3, dtype=torch.int8, device=DEV)
    sum_scale = torch.full((L, pool, H), 5.0, device=DEV)
    want_sum, want_sum_scale = np.full((L, pool, H, D), 3, dtype=np.int8), np.full((L, pool, H), 5.0)
    kw = dict(tokens_before=i32(before), chunk_tokens=i32(tokens), k_sum=sums, k_sum_scale=sum_scale, status=status)
    if c.get("packed"):
        base = np.cumsum([0] + tokens[:-1])
        packed = torch.cat([xt[:, i, :, :t] for i, t in enumerate(tokens)], dim=2)
        km.append_paged8(packed[0], packed[1], kc, vc, ks, vs, i32(table), n_tokens=n, row_base=i32(base), **kw)
    else:
        km.append_paged8(xt[0], xt[1], kc, vc, ks, vs, i32(table), **kw)
    torch.cuda.synchronize()
    for l in range(L):
        ref_tokens = [min(t, max(0, table.shape[1] * page - b)) for b, t in zip(before, tokens)]
        ref.append([xv[0, i, l] for i in range(C)], kb[l], ksv[l], table, before, ref_tokens, page,
                   sums=(want_sum[l], want_sum_scale[l]))
        ref.append([xv[1, i, l] for i in range(C)], vb[l], vsv[l], table, before, ref_tokens, page)
    np.testing.assert_array_equal(ks.cpu().double().numpy(), ksv)
    np.testing.assert_array_equal(vs.cpu().double().numpy(), vsv)
    for got, want in ((kc, kb), (vc, vb)):
        g, w = got.cpu().numpy(), want
        both_nan = ((g & 0x7F) == 0x7F) & ((w & 0x7F) == 0x7F)
        assert ((g == w) | both_nan).all(), int(((g != w) & ~both_nan).sum())
    np.testing.assert_array_equal(sums.cpu().numpy(), want_sum)
    np.testing.assert_array_equal(sum_scale.cpu().double().numpy(), want_sum_scale)
    assert int(status) == (km.STATUS_BAD_PAGE if c.get("bad") else km.STATUS_BAD_LENGTH if c.get("cut") else 0)


@pytest.mark.parametrize("first", [0, 3, 6])
def test_append_ends_where_a_view_of_the_table_does(first):
    """Two columns of a wider table: chunks that outgrow them are cut and flagged, as with a copy of the columns,
    and no page that only the other columns name is written."""
    rng = np.random.default_rng(23)
    before, tokens, page, H, D = [20, 5, 10], [32, 30, 6], 16, 2, 128
    pool = 3 * 8 + 1
    whole = i32(rng.permutation(pool)[:24].reshape(3, 8))
    xt, _ = bf16(rng.standard_normal((2, 3, 1, 32, H, D)))
    kept = [new_cache(rng, 1, pool, page, H, D, "heads") for _ in range(2)]
    got = []
    for view in (whole[:, first:first + 2], whole[:, first:first + 2].contiguous()):
        (kc, ks), (vc, vs) = [(k[0].clone(), k[2].clone()) for k in kept]
        status = i32([0])
        km.append_paged8(xt[0], xt[1], kc, vc, ks, vs, view, tokens_before=i32(before), chunk_tokens=i32(tokens),
                         status=status)
        got.append((kc, vc, ks, vs))
        assert int(status) == km.STATUS_BAD_LENGTH
    for a, b in zip(*got):
        assert torch.equal(a, b)
    mine = set(whole[:, first:first + 2].flatten().tolist())
    others = [p for p in range(pool) if p not in mine]
    for (kc, _, ks, _), (now, now_scale) in zip(kept, (got[0][0::2], got[0][1::2])):
        assert torch.equal(now[:, others], kc[:, others]) and torch.equal(now_scale[:, others], ks[:, others])


def test_append_in_steps_equals_append_at_once():
    """One token at a time and all at once leave the same bytes where the largest magnitude comes first, and
    the same values up to the roundings of a lift otherwise."""
    rng = np.random.default_rng(11)
    H, D, page, n = 2, 128, 16, 40
    x = rng.standard_normal((1, 1, n, H, D))
    x[:, :, ::page] *= 8
    xt, _ = bf16(x)
    table, pool = table_for(rng, [n], page)
    one, many = km.Cache8.allocate(1, pool, page, H, D), km.Cache8.allocate(1, pool, page, H, D)
    km.append_paged8(xt, xt, one.k, one.v, one.k_scale, one.v_scale, i32(table), k_sum=one.k_sum,
                     k_sum_scale=one.k_sum_scale)
    for t in range(n):
        km.append_paged8(xt[:, :, t:t + 1], xt[:, :, t:t + 1], many.k, many.v, many.k_scale, many.v_scale, i32(table),
                         tokens_before=i32([t]), k_sum=many.k_sum, k_sum_scale=many.k_sum_scale)
    torch.cuda.synchronize()
    for a, b in ((one.k, many.k), (one.v, many.v)):
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
    assert torch.equal(one.k_scale, many.k_scale) and torch.equal(one.k_sum, many.k_sum)
    assert torch.equal(one.k_sum_scale, many.k_sum_scale)


# ---------------------------------------------------------------------------
# page selection
# ---------------------------------------------------------------------------

SELECT_CASES = {
    "few_pages": dict(kv=[1, 0, 16, 17, 64], keep=4),
    "plain": dict(kv=[700, 1000, 333], keep=9, first=1, last=2),
    "keep_two": dict(kv=[700, 40], keep=2),
    "group1": dict(kv=[500], keep=7, H=4, G=1),
    "group20": dict(kv=[500, 300], keep=7, H=2, G=20, first=0, last=1),
    "group64": dict(kv=[500], keep=7, H=1, G=64),
    "d64": dict(kv=[900, 260], keep=6, D=64, H=3, G=5),
    "page64": dict(kv=[5000, 4097], keep=11, page=64),
    "ties": dict(kv=[1600], keep=20, ties=True),
    "all_equal": dict(kv=[3000], keep=33, equal=True),
    "zero_query": dict(kv=[900], keep=5, zero=True),
    "nonfinite_query": dict(kv=[900], keep=5, nonfinite=True),
    "bad_page": dict(kv=[900], keep=50, bad=True),
    "long": dict(kv=[40000], keep=100, H=1),
    "most_pages": dict(kv=[140001, 16 * 8192 + 1], keep=77, H=1, G=2, D=64),
    "most_pages_ties": dict(kv=[140001], keep=500, H=1, G=2, D=64, ties=True),
}


@pytest.mark.parametrize("name", sorted(SELECT_CASES))
def test_select(name):
    c = SELECT_CASES[name]
    rng = np.random.default_rng(13)
    kv, keep, page = c["kv"], c["keep"], c.get("page", 16)
    H, G, D, first, last = c.get("H", 2), c.get("G", 4), c.get("D", 128), c.get("first", 1), c.get("last", 1)
    table, pool = table_for(rng, kv, page)
    if c.get("bad"):
        table[0, 5] = -1
        table[0, 20] = pool + 3
    k_sum = rng.integers(-127, 128, size=(pool, H, D)).astype(np.int8)
    scale = 2.0 ** rng.integers(-3, 3, size=(pool, H))
    if c.get("ties"):
        k_sum[:] = k_sum[rng.integers(0, 4, size=pool)]
        scale[:] = 0.5
    if c.get("equal"):
        k_sum[:], scale[:] = 1, 2.0
    x = rng.standard_normal((len(kv), H * G, D)) * 3
    if c.get("zero"):
        x[:] = 0
    if c.get("nonfinite"):
        x[rng.random(x.shape) < 0.05] = np.nan
        x[rng.random(x.shape) < 0.05] = -np.inf
    qt, qv = bf16(x)
    sel = torch.full((len(kv), H, keep), -9, dtype=torch.int32, device=DEV)
    count, status = i32(np.full((len(kv), H), -9)), i32([0])
    km.select_pages(qt, torch.tensor(k_sum, device=DEV), torch.tensor(scale, dtype=torch.float32, device=DEV),
                    i32(table), i32(kv), sel, count, n_keys=max(kv), page_size=page, n_first=first, n_last=last,
                    status=status)
    torch.cuda.synchronize()
    want = ref.select(qv, k_sum, scale, table, kv, page, keep, first, last)
    sel, count = sel.cpu().numpy(), count.cpu().numpy()
    for r in range(len(kv)):
        for h in range(H):
            w = want[r * H + h]
            assert count[r, h] == len(w)
            assert list(sel[r, h, :len(w)]) == w
            assert (sel[r, h, len(w):] == -1).all()
    assert int(status) == (km.STATUS_BAD_PAGE if c.get("bad") else 0)


@pytest.mark.parametrize("G", [3, 20])
@pytest.mark.parametrize("D", [64, 128])
def test_select_most_pages_of_many_requests(G, D):
    """Over 8192 pages a request, scored by the workgroup that selects: more than 128 (request, KV head) pairs."""
    rng = np.random.default_rng(31)
    kv, keep, H = [0] * 63 + [16 * km.MAX_SELECT_PAGES, 200000], 40, 2
    table, pool = table_for(rng, kv, 16)
    k_sum = rng.integers(-127, 128, size=(pool, H, D)).astype(np.int8)
    scale = 2.0 ** rng.integers(-3, 3, size=(pool, H))
    qt, qv = bf16(rng.standard_normal((65, H * G, D)))
    sel, count = i32(np.full((65, H, keep), -9)), i32(np.full((65, H), -9))
    km.select_pages(qt, torch.tensor(k_sum, device=DEV), torch.tensor(scale, dtype=torch.float32, device=DEV),
                    i32(table), i32(kv), sel, count, n_keys=max(kv), page_size=16)
    torch.cuda.synchronize()
    want = ref.select(qv[63:], k_sum, scale, table[63:], kv[63:], 16, keep, 1, 1)
    assert sel[63:].reshape(2 * H, keep).tolist() == want and (count[63:] == keep).all()
    assert (sel[:63] == -1).all() and (count[:63] == 0).all()


@pytest.mark.parametrize("pages", [60, 300, 1100])
def test_select_scores_that_are_not_numbers(pages):
    """Pages whose sums were never formed: any NaN as their scale (with any bits) ranks them last, and neither
    adds to the selection nor leaves a place of it open.  300 pages in one kernel, 1100 in two."""
    rng = np.random.default_rng(29)
    kv, keep, H, G, D = [16 * pages, 16 * pages - 9], 9, 2, 4, 128
    table, pool = table_for(rng, kv, 16)
    k_sum = rng.integers(-127, 128, size=(pool, H, D)).astype(np.int8)
    scale = (2.0 ** rng.integers(-3, 3, size=(pool, H))).astype(np.float32)
    qt, qv = bf16(rng.standard_normal((2, H * G, D)))
    for share in (0.3, 1.0):
        bits = scale.copy().view(np.uint32)
        lost = rng.random(pool) < share
        bits[lost] = rng.choice(np.array([0x7FFFFFFF, 0xFFFFFFFF, 0x7FC00000, 0xFFC00000, 0x7F800001], dtype=np.uint32),
                                size=bits[lost].shape)
        sel = torch.full((4, H, keep), -9, dtype=torch.int32, device=DEV)      # two rows more than the call's
        count = i32(np.full((2, H), -9))
        km.select_pages(qt, torch.tensor(k_sum, device=DEV), torch.tensor(bits.view(np.int32), device=DEV).view(torch.float32),
                        i32(table), i32(kv), sel[1:3], count, n_keys=max(kv), page_size=16)
        torch.cuda.synchronize()
        # ranked as a page that is not in the pool
        known = np.where(lost[np.maximum(table, 0)], -1, table)
        want = ref.select(qv, k_sum, scale.astype(float), known, kv, 16, keep, 1, 1)
        assert sel[1:3].reshape(2 * H, keep).tolist() == want
        assert (count == keep).all() and (sel[0] == -9).all() and (sel[3] == -9).all()


def test_select_without_keys():
    """No request has a key: nothing is selected, and nothing of the tables is looked at."""
    q = torch.zeros((3, 8, 128), dtype=torch.bfloat16, device=DEV)
    sel, count = i32(np.full((3, 2, 4), -9)), i32(np.full((3, 2), -9))
    km.select_pages(q, torch.zeros((5, 2, 128), dtype=torch.int8, device=DEV), torch.ones((5, 2), device=DEV),
                    i32(np.full((3, 1), 99)), i32([0, 7, 300]), sel, count, n_keys=0, page_size=16)
    torch.cuda.synchronize()
    assert (sel == -1).all() and (count == 0).all()


def test_select_zeros_of_either_sign_tie():
    """A negative sum under a scale of zero is a score of -0, which is no less than 0."""
    k_sum = np.full((40, 1, 64), 1, dtype=np.int8)
    k_sum[::2] = -1
    scale, table = np.zeros((40, 1)), np.arange(40)[None].astype(np.int32)
    qt, qv = bf16(np.ones((1, 4, 64)))
    sel, count = i32(np.full((1, 1, 10), -9)), i32([[-9]])
    km.select_pages(qt, torch.tensor(k_sum, device=DEV), torch.tensor(scale, dtype=torch.float32, device=DEV),
                    i32(table), i32([640]), sel, count, n_keys=640, page_size=16)
    torch.cuda.synchronize()
    assert sel.flatten().tolist() == ref.select(qv, k_sum, scale, table, [640], 16, 10, 1, 1)[0] == [*range(9), 39]


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

ATTEND_CASES = {
    # lengths around parts, steps and pages; empty requests
    "lengths": dict(kv=[0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300]),
    "lengths_bf16": dict(kv=[0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300], cache="bf16"),
    "d64": dict(kv=[5, 90, 200], D=64, H=3, G=5),
    "d64_bf16": dict(kv=[5, 90, 200], D=64, H=3, G=5, cache="bf16"),
    "mha": dict(kv=[40, 129], H=6, G=1, cache="bf16"),
    "mqa": dict(kv=[77, 130], H=1, G=16),
    "group7": dict(kv=[77, 130], H=2, G=7),
    "group40": dict(kv=[77, 130], H=1, G=40),
    "group64": dict(kv=[50, 66], H=1, G=64, nq=[1, 1]),
    # several queries: rows that see no key, ragged, padding rows untouched
    "spec": dict(kv=[100, 3, 0, 64], nq=[4, 5, 2, 5], H=2, G=4),
    "spec_bf16": dict(kv=[100, 3, 0, 64], nq=[4, 5, 2, 5], H=2, G=4, cache="bf16", packed=True),
    "prompt": dict(kv=[100, 40, 200], nq=[100, 33, 70], H=2, G=4, packed=True),
    "prompt_d64": dict(kv=[100, 40, 200], nq=[100, 33, 70], H=2, G=3, D=64, packed=True),
    "prompt_bf16": dict(kv=[190, 64, 130], nq=[64, 64, 1], H=1, G=7, cache="bf16", packed=True, page=48),
    "prompt_d64_bf16": dict(kv=[190, 64, 130], nq=[64, 64, 1], H=1, G=7, D=64, cache="bf16", packed=True, page=32),
    "prompt_more_queries_than_keys": dict(kv=[10, 70], nq=[50, 90], H=1, G=8, packed=True),
    "prompt_no_queries": dict(kv=[10, 70], nq=[0, 40], H=1, G=8, packed=True),
    "not_causal": dict(kv=[50, 129, 0], nq=[20, 3, 40], H=1, G=8, causal=False),
    "not_causal_bf16": dict(kv=[50, 129, 0], nq=[20, 3, 40], H=2, G=4, causal=False, cache="bf16"),
    "window": dict(kv=[200, 90, 10], window=33),
    "window_one": dict(kv=[200, 90, 10], window=1, nq=[5, 1, 10], H=1, G=4),
    "window_prompt": dict(kv=[300, 130], nq=[128, 100], window=40, H=2, G=4, packed=True),
    "window_prompt_bf16": dict(kv=[300, 130], nq=[128, 100], window=64, H=1, G=4, packed=True, cache="bf16"),
    # pages
    "page32": dict(kv=[100, 31, 33], page=32),
    "page64": dict(kv=[100, 63, 65], page=64, nq=[3, 3, 3]),
    "page48": dict(kv=[100, 47, 49], page=48, cache="bf16"),
    "page16_rows": dict(kv=[100, 63, 65], layout="slots"),
    "bad_pages": dict(kv=[100, 80], bad=[(0, 2), (1, 0), (1, 4)], page=16),
    "bad_pages_prompt": dict(kv=[150, 80], nq=[70, 70], H=1, G=4, bad=[(0, 2), (1, 0), (1, 4)], page=16),
    "all_bad": dict(kv=[40], bad=[(0, 0), (0, 1), (0, 2)]),
    # splits
    "split2": dict(kv=[300, 1, 0, 64], splits=2),
    "split7": dict(kv=[700, 33, 250], splits=7, nq=[2, 2, 2], lse=True),
    "split512": dict(kv=[300], splits=512),
    "split_prompt": dict(kv=[300, 90], nq=[90, 64], H=1, G=4, splits=3),
    "split_prompt_bf16": dict(kv=[300, 90], nq=[90, 64], H=1, G=4, splits=5, cache="bf16", window=100),
    "long": dict(kv=[9000], H=1, G=8),
    "long_prompt": dict(kv=[3000], nq=[40], H=1, G=8),
    # values
    "large_scores": dict(kv=[200, 90], scale=4.0),
    "negative_scale": dict(kv=[200, 90], scale=-0.3),
    "zero_scale": dict(kv=[200], scale=0.0),
}


def attend_case(c, seed=17):
    rng = np.random.default_rng(seed)
    kv = c["kv"]
    R = len(kv)
    nq = c.get("nq", [1] * R)
    page, H, G, D = c.get("page", 16), c.get("H", 2), c.get("G", 8), c.get("D", 128)
    packed = c.get("packed", False)
    table, pool = table_for(rng, kv, page)
    for r, j in c.get("bad", ()):
        table[r, j] = -1 if j % 2 else pool + 1
    n_max = max(max(nq), 1)
    base = np.cumsum([0] + list(nq[:-1])) + 2 if packed else np.arange(R) * n_max
    rows = int(sum(nq)) + 5 if packed else R * n_max
    qt, qv = bf16(rng.standard_normal((rows, H * G, D)))
    if c.get("cache") == "bf16":
        planes = [bf16(rng.standard_normal((pool, page, H, D))) for _ in range(2)]
        k, v = planes[0][1], planes[1][1]
        kt, vt = planes[0][0], planes[1][0]
        scales = {}
        # unused slots hold NaN
        hole = torch.tensor(~used_slots(table, kv, page, pool), device=DEV)
        for t in (kt, vt):
            t[hole] = float("nan")
    else:
        out = []
        for layout in (c.get("layout", "heads"), "dense"):
            x = rng.standard_normal((pool, page, H, D)) * 50
            b = ref.encode(x)
            b[~used_slots(table, kv, page, pool)] = 0x7F
            e = rng.integers(-7, -4, size=(pool, H))
            t = torch.tensor(b, device=DEV)
            if layout == "heads":
                t = t.transpose(1, 2).contiguous().transpose(1, 2)
            elif layout == "slots":
                w = torch.full((pool, page, H + 2, D), 0x7F, dtype=torch.uint8, device=DEV)
                w[:, :, 1:H + 1] = t
                t = w[:, :, 1:H + 1]
            out.append((t, ref.decode(b) * 2.0 ** e[:, None, :, None],
                        torch.tensor(2.0 ** e, dtype=torch.float32, device=DEV)))
        (kt, k, ks), (vt, v, vs) = out
        scales = dict(k_scale=ks, v_scale=vs)
    return dict(kv=kv, nq=nq, page=page, H=H, G=G, D=D, table=table, pool=pool, base=base, rows=rows, q=qt, qv=qv,
                kt=kt, vt=vt, k=k, v=v, scales=scales, packed=packed, n_max=n_max)


def used_slots(table, kv, page, pool):
    used = np.zeros((pool, page), dtype=bool)
    for r, n in enumerate(kv):
        for t in range(n):
            pg = int(table[r, t // page])
            if 0 <= pg < pool:
                used[pg, t % page] = True
    return used


def check_attend(out, lse, s, scale, causal=True, window=0, sel=None, filler=-7.0):
    a = (s["qv"], s["k"], s["v"], s["table"], s["kv"], s["nq"], s["base"], s["page"], scale, causal, window, sel)
    want, want_lse = ref.attend(*a)
    size, _ = ref.attend(s["qv"], s["k"], np.abs(s["v"]), *a[3:])
    mine = ~np.isnan(want_lse)
    got = out.double().cpu().numpy()
    assert np.isfinite(got[mine]).all()
    bound = BOUND * size
    bad = np.abs(got - want) > bound
    assert not bad[mine].any(), (int(bad[mine].sum()), float(np.max((np.abs(got - want) / (size + 1e-30))[mine])))
    assert (got[~mine] == filler).all()
    if lse is not None:
        g = lse.double().cpu().numpy()
        empty = mine & np.isneginf(want_lse)
        assert np.isneginf(g[empty]).all()
        full = mine & ~np.isneginf(want_lse)
        tol = 2.0 ** -11 * np.maximum(1.0, np.abs(want_lse[full]) / 16)
        assert (np.abs(g[full] - want_lse[full]) <= tol).all()
        assert (g[~mine] == filler).all()


@pytest.mark.parametrize("name", sorted(ATTEND_CASES))
def test_attend(name):
    c = ATTEND_CASES[name]
    s = attend_case(c)
    out = torch.full_like(s["q"], -7.0)
    lse = torch.full(s["q"].shape[:2], -7.0, device=DEV)
    status = i32([0])
    scale = c.get("scale", s["D"] ** -0.5)
    km.attend_paged(s["q"], s["kt"], s["vt"], out, i32(s["table"]), i32(s["kv"]), n_queries=s["n_max"],
                    n_keys=max(max(s["kv"]), 1), q_base=i32(s["base"]) if s["packed"] else None,
                    q_tokens=i32(s["nq"]), scale=scale, causal=c.get("causal", True), window=c.get("window", 0),
                    lse=lse, n_splits=c.get("splits", 0), status=status, **s["scales"])
    torch.cuda.synchronize()
    check_attend(out, lse, s, scale, c.get("causal", True), c.get("window", 0))
    assert int(status) == (km.STATUS_BAD_PAGE if c.get("bad") else 0)


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("nq", [[1, 1, 1], [3, 0, 5], [40, 70, 1]])
@pytest.mark.parametrize("splits", [8, 9, 65])
def test_attend_many_parts_of_small_heads(cache, nq, splits):
    s = attend_case(dict(kv=[700, 33, 1500], nq=nq, H=3, G=2, D=64, cache=cache))
    out, lse = torch.full_like(s["q"], -7.0), torch.full(s["q"].shape[:2], -7.0, device=DEV)
    km.attend_paged(s["q"], s["kt"], s["vt"], out, i32(s["table"]), i32(s["kv"]), n_queries=s["n_max"], n_keys=1500,
                    q_tokens=i32(nq), lse=lse, n_splits=splits, **s["scales"])
    torch.cuda.synchronize()
    check_attend(out, lse, s, 64 ** -0.5)


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("kv,nq", [([10, 3, 70], [16, 12, 16]), ([10, 70], [50, 90])])
def test_attend_longest_window(cache, kv, nq):
    """A window of the type's largest value is no window, also for queries before the first key."""
    s = attend_case(dict(kv=kv, nq=nq, H=2, G=1 if max(nq) <= 16 else 4, cache=cache))
    outs = []
    for window in (0, 2 ** 31 - 1):
        out = torch.full_like(s["q"], -7.0)
        km.attend_paged(s["q"], s["kt"], s["vt"], out, i32(s["table"]), i32(kv), n_queries=s["n_max"], n_keys=max(kv),
                        q_tokens=i32(nq), window=window, **s["scales"])
        outs.append(out)
    torch.cuda.synchronize()
    assert torch.equal(*outs)


POISON_CASES = {
    "spec": dict(kv=[40, 70], nq=[4, 6], H=2, G=2),
    "spec_bf16": dict(kv=[40, 70], nq=[4, 6], H=2, G=2, cache="bf16"),
    "prompt": dict(kv=[100, 200], nq=[60, 70], H=1, G=4),
    "prompt_bf16": dict(kv=[100, 200], nq=[60, 70], H=1, G=4, cache="bf16"),
    "prompt_window": dict(kv=[100, 200], nq=[60, 70], H=1, G=4, window=40),
    "prompt_window_bf16": dict(kv=[100, 200], nq=[60, 70], H=1, G=4, window=40, cache="bf16"),
    "prompt_d64": dict(kv=[100, 200], nq=[60, 70], H=1, G=4, D=64),
    "prompt_d64_bf16": dict(kv=[100, 200], nq=[60, 70], H=1, G=4, D=64, cache="bf16", window=50),
}


@pytest.mark.parametrize("name", sorted(POISON_CASES))
def test_attend_values_that_a_row_does_not_see(name):
    """NaN (and infinities in bf16) in a token's K and V reach the rows that see it, as NaN, and no others."""
    c = POISON_CASES[name]
    s = attend_case(c)
    when = [s["kv"][0] - 2, s["kv"][1] - s["nq"][1] // 2]
    for r, t in enumerate(when):
        pg, at = int(s["table"][r, t // s["page"]]), t % s["page"]
        for val, (tt, vals) in ((np.nan, (s["kt"], s["k"])), (np.inf, (s["vt"], s["v"]))):
            if c.get("cache") == "bf16":
                tt[pg, at, :, 3::7] = val
                vals[pg, at, :, 3::7] = val
            else:
                tt[pg, at, :, 3::7] = 0x7F
                vals[pg, at, :, 3::7] = np.nan
    out = torch.full_like(s["q"], -7.0)
    scale = s["D"] ** -0.5
    km.attend_paged(s["q"], s["kt"], s["vt"], out, i32(s["table"]), i32(s["kv"]), n_queries=s["n_max"],
                    n_keys=max(s["kv"]), q_tokens=i32(s["nq"]), window=c.get("window", 0), **s["scales"])
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    want, _ = ref.attend(s["qv"], s["k"], s["v"], s["table"], s["kv"], s["nq"], s["base"], s["page"], scale, True,
                         c.get("window", 0))
    size, _ = ref.attend(s["qv"], s["k"], np.abs(s["v"]), s["table"], s["kv"], s["nq"], s["base"], s["page"], scale,
                         True, c.get("window", 0))
    for r, t in enumerate(when):
        first = s["kv"][r] - s["nq"][r]
        for i in range(s["nq"][r]):
            row = int(s["base"][r]) + i
            sees = t <= first + i and (not c.get("window") or t > first + i - c["window"])
            if sees:
                assert np.isnan(got[row]).all()
            else:
                assert (np.abs(got[row] - want[row]) <= BOUND * size[row]).all(), (r, i)


@pytest.mark.parametrize("nq,window", [([1, 1, 1], 0), ([4, 5, 2], 20), ([70, 40, 70], 0), ([70, 40, 70], 40)])
@pytest.mark.parametrize("D", [64, 128])
def test_attend_scales_of_pages_that_no_request_has(nq, window, D):
    """The scales of a page that is nobody's, the pool's first, may hold anything."""
    s = attend_case(dict(kv=[100, 45, 190], nq=nq, H=2, G=2, D=D, bad=[(0, 2)]))
    first = {k: torch.cat([torch.full_like(t[:1], 0x7F if t.dtype is torch.uint8 else 1.0), t])
             for k, t in dict(k_cache=s["kt"], v_cache=s["vt"], **s["scales"]).items()}
    table, outs = i32(np.where(s["table"] >= 0, s["table"] + 1, -1)), []
    for scale in (1.0, float("nan"), float("inf"), 0.0, -float("inf")):
        first["k_scale"][0] = first["v_scale"][0] = scale
        out, lse = torch.full_like(s["q"], -7.0), torch.full(s["q"].shape[:2], -7.0, device=DEV)
        km.attend_paged(s["q"], out=out, page_table=table, kv_tokens=i32(s["kv"]), n_queries=max(nq), n_keys=190,
                        q_tokens=i32(nq), window=window, lse=lse, **first)
        outs.append((out, lse))
    torch.cuda.synchronize()
    check_attend(*outs[0], s, D ** -0.5, True, window)
    for out, lse in outs[1:]:
        assert torch.equal(out, outs[0][0]) and torch.equal(lse, outs[0][1])


def test_attend_clean_keys_poisoned_values():
    """A value that is not finite, under finite scores: only its columns, only in the rows that see it."""
    for cache in ("e4m3", "bf16"):
        for nq, D in (([4], 128), ([70], 128), ([70], 64)):
            s = attend_case(dict(kv=[90], nq=nq, H=1, G=4, D=D, cache=cache))
            t = 90 - nq[0] // 2
            pg, at = int(s["table"][0, t // 16]), t % 16
            if cache == "bf16":
                s["vt"][pg, at, :, 5] = float("inf")
                s["v"][pg, at, :, 5] = np.inf
            else:
                s["vt"][pg, at, :, 5] = 0x7F
                s["v"][pg, at, :, 5] = np.nan
            out = torch.full_like(s["q"], -7.0)
            km.attend_paged(s["q"], s["kt"], s["vt"], out, i32(s["table"]), i32([90]), n_queries=nq[0], n_keys=90,
                            **s["scales"])
            torch.cuda.synchronize()
            got = out.double().cpu().numpy()
            v = s["v"].copy()
            v[~np.isfinite(v)] = 0.0
            a = (s["table"], [90], nq, s["base"], 16, D ** -0.5)
            want, _ = ref.attend(s["qv"], s["k"], v, *a)
            size, _ = ref.attend(s["qv"], s["k"], np.abs(v), *a)
            sees = np.arange(nq[0]) + 90 - nq[0] >= t
            col = np.zeros(D, dtype=bool)
            col[5] = True
            hit = sees[:, None, None] & col[None, None, :] & np.ones((1, 4, 1), dtype=bool)
            assert not np.isfinite(got[hit]).any()
            ok = np.abs(got - want) <= BOUND * size
            assert ok[~hit].all()


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nq,window", [(4, 0), (70, 0), (70, 50)])
@pytest.mark.parametrize("splits", [2, 3, 7])
def test_attend_poisoned_values_in_split_work(cache, D, nq, window, splits):
    """As with whole work: a value that is not finite goes to its column of the rows that see it, whichever part
    of the keys holds it, and to nothing else.  Two in different tiles."""
    s = attend_case(dict(kv=[300, 150], nq=[nq, nq], H=2, G=4, D=D, cache=cache))
    cols, when = (5, D - 3), [(0, 300 - nq // 2), (0, 300 - nq), (1, 150 - 2)]
    for (r, t), col in zip(when, (cols[0], cols[1], cols[0])):
        pg, at = int(s["table"][r, t // 16]), t % 16
        s["vt"][pg, at, :, col] = float("inf") if cache == "bf16" else 0x7F
        s["v"][pg, at, :, col] = 0.0
    out = torch.full_like(s["q"], -7.0)
    km.attend_paged(s["q"], s["kt"], s["vt"], out, i32(s["table"]), i32(s["kv"]), n_queries=nq, n_keys=300,
                    window=window, n_splits=splits, **s["scales"])
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    v = np.where(np.isfinite(s["v"]), s["v"], 0.0)            # slots that no request uses hold NaN
    a = (s["table"], s["kv"], s["nq"], s["base"], 16, D ** -0.5, True, window)
    want, size = ref.attend(s["qv"], s["k"], v, *a)[0], ref.attend(s["qv"], s["k"], np.abs(v), *a)[0]
    hit = np.zeros(got.shape, dtype=bool)
    for (r, t), col in zip(when, (cols[0], cols[1], cols[0])):
        at = s["kv"][r] - nq + np.arange(nq)
        sees = (t <= at) & (t > at - window if window else True)
        hit[r * nq:(r + 1) * nq, :, col] |= sees[:, None]
    assert not np.isfinite(got[hit]).any()
    assert (np.abs(got - want) <= BOUND * size)[~hit].all()


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("splits", [1, 2])
def test_attend_poisoned_value_in_a_selected_page(cache, splits):
    """The last page, seen in part, with a value that is not finite in a token that is seen and one in a token
    that is not; a page that is not selected is full of them."""
    s = attend_case(dict(kv=[200, 90], H=2, G=4, cache=cache))
    sel, count = i32(np.tile([[[1, 3, 12]], [[0, 2, 5]]], (1, 2, 1))), i32(np.full((2, 2), 3))
    odd = float("inf") if cache == "bf16" else 0x7F
    for r, n in enumerate(s["kv"]):
        last = int(s["table"][r, (n - 1) // 16])
        s["vt"][last, (n - 1) % 16, :, 7] = odd
        s["vt"][last, n % 16, :, 9] = odd
        s["vt"][int(s["table"][r, 4])] = odd
        s["v"][last, (n - 1) % 16, :, 7] = 0.0
    v = np.where(np.isfinite(s["v"]), s["v"], 0.0)
    out = torch.full_like(s["q"], -7.0)
    km.attend_paged(s["q"], s["kt"], s["vt"], out, i32(s["table"]), i32(s["kv"]), n_queries=1, n_keys=200, sel=sel,
                    sel_count=count, n_splits=splits, **s["scales"])
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    a = (s["table"], s["kv"], s["nq"], s["base"], 16, 128 ** -0.5, True, 0, [[1, 3, 12]] * 2 + [[0, 2, 5]] * 2)
    want, size = ref.attend(s["qv"], s["k"], v, *a)[0], ref.attend(s["qv"], s["k"], np.abs(v), *a)[0]
    hit = np.zeros(got.shape, dtype=bool)
    hit[:, :, 7] = True
    assert not np.isfinite(got[hit]).any()
    assert (np.abs(got - want) <= BOUND * size)[~hit].all()


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("page", [16, 64])
def test_attend_selected_pages(cache, page):
    s = attend_case(dict(kv=[900, 40, 0, 1000], H=2, G=4, cache=cache, page=page))
    keep = 6
    sel, sel_list = np.full((4, 2, keep), -1, dtype=np.int32), []
    rng = np.random.default_rng(5)
    for r, n in enumerate(s["kv"]):
        for h in range(2):
            pages = -(-n // page)
            pick = sorted(rng.permutation(pages)[:keep].tolist())
            if pages and pages - 1 not in pick:
                pick = sorted(pick[1:] + [pages - 1])
            sel[r, h, :len(pick)] = pick
            sel_list.append(pick)
    count = (sel >= 0).sum(-1)
    for splits in (0, 1, 3):
        out = torch.full_like(s["q"], -7.0)
        lse = torch.full(s["q"].shape[:2], -7.0, device=DEV)
        km.attend_paged(s["q"], s["kt"], s["vt"], out, i32(s["table"]), i32(s["kv"]), n_queries=1, n_keys=1000,
                        sel=i32(sel), sel_count=i32(count), lse=lse, n_splits=splits, **s["scales"])
        torch.cuda.synchronize()
        check_attend(out, lse, s, 128 ** -0.5, sel=sel_list)


def test_selected_pages_end_where_a_view_of_the_table_does():
    """An index past the view's columns names no page, whatever the tensor behind it holds there."""
    s = attend_case(dict(kv=[300, 300], H=2, G=4))
    whole, kv = i32(s["table"]), i32(s["kv"])
    sel, count = i32(np.tile([0, 3, 9, 12], (2, 2, 1))), i32(np.full((2, 2), 4))
    inside = [[0, 3]] * 4
    for first in (0, 5):
        view = whole[:, first:first + 9]
        part = dict(s, table=s["table"][:, first:first + 9])
        for table in (view, view.contiguous()):
            out, status = torch.full_like(s["q"], -7.0), i32([0])
            km.attend_paged(s["q"], s["kt"], s["vt"], out, table, kv, n_queries=1, n_keys=300, sel=sel,
                            sel_count=count, status=status, **s["scales"])
            torch.cuda.synchronize()
            assert int(status) == km.STATUS_BAD_PAGE
            check_attend(out, None, part, 128 ** -0.5, sel=inside)


def test_attend_strided_rows_and_lse():
    """Queries inside a wider projection, outputs with a gap between rows, a transposed lse."""
    s = attend_case(dict(kv=[120, 33], nq=[3, 3], H=2, G=4))
    wide = torch.zeros((6, 8 + 4, 128), dtype=torch.bfloat16, device=DEV)
    wide[:, 2:10] = s["q"]
    room = torch.full((6, 11, 128), -7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((8, 6), -7.0, device=DEV)
    km.attend_paged(wide[:, 2:10], s["kt"], s["vt"], room[:, 1:9], i32(s["table"]), i32(s["kv"]), n_queries=3,
                    n_keys=120, lse=lse.t(), **s["scales"])
    torch.cuda.synchronize()
    check_attend(room[:, 1:9].contiguous(), lse.t().contiguous(), s, 128 ** -0.5)
    assert (room[:, 0] == -7.0).all() and (room[:, 9:] == -7.0).all()


def test_attend_scores_of_any_size():
    """Scores far outside the range of exp: the softmax is their difference's alone."""
    s = attend_case(dict(kv=[100], H=1, G=8))
    for scale in (3000.0, -3000.0):
        out = torch.zeros_like(s["q"])
        lse = torch.zeros(s["q"].shape[:2], device=DEV)
        km.attend_paged(s["q"], s["kt"], s["vt"], out, i32(s["table"]), i32([100]), n_queries=1, n_keys=100,
                        scale=scale, lse=lse, **s["scales"])
        torch.cuda.synchronize()
        pos = [int(s["table"][0, t // 16]) * 16 + t % 16 for t in range(100)]
        k, v = s["k"].reshape(-1, 128)[pos], s["v"].reshape(-1, 128)[pos]
        best = (s["qv"][0] @ k.T) * scale
        for g in range(8):
            order = np.argsort(best[g])
            assert best[g][order[-1]] - best[g][order[-2]] > 50            # one key takes everything
            got = out[0, g].double().cpu().numpy()
            assert (np.abs(got - v[order[-1]]) <= 2.0 ** -8 * np.abs(v[order[-1]])).all()
            assert abs(float(lse[0, g]) / best[g].max() - 1) < 1e-5


def test_attend_repeats_bit_for_bit():
    s = attend_case(dict(kv=[3000, 700, 1500], nq=[3, 3, 3], H=2, G=4))
    got = []
    for _ in range(3):
        out = torch.zeros_like(s["q"])
        km.attend_paged(s["q"], s["kt"], s["vt"], out, i32(s["table"]), i32(s["kv"]), n_queries=3, n_keys=3000,
                        **s["scales"])
        got.append(out.view(torch.int16).clone())
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_cache_offsets_past_32_bits():
    """Pages that lie more than 4 GiB apart: append, then attention over them."""
    page, H, D, far = 16, 1, 128, (1 << 32) + (1 << 20)
    buf = torch.empty(2 * far + (1 << 20), dtype=torch.uint8, device=DEV)

    def view(offset):
        return torch.as_strided(buf, (1, 3, page, H, D), (0, far, D, page * D, 1), offset)

    kc, vc = view(0), view(1 << 16)
    scales = [torch.ones((1, 3, H), device=DEV) for _ in range(2)]
    rng = np.random.default_rng(2)
    xt, _ = bf16(rng.standard_normal((2, 1, 1, 40, H, D)))
    table = i32([[2, 0, 1]])
    km.append_paged8(xt[0], xt[1], kc, vc, scales[0], scales[1], table)
    near = km.Cache8.allocate(1, 3, page, H, D)
    km.append_paged8(xt[0], xt[1], near.k, near.v, near.k_scale, near.v_scale, table)
    q, _ = bf16(rng.standard_normal((1, 8, D)))
    outs = []
    for k, v, ks, vs in ((kc[0], vc[0], scales[0][0], scales[1][0]), (near.k[0], near.v[0], near.k_scale[0],
                                                                     near.v_scale[0])):
        out = torch.zeros_like(q)
        km.attend_paged(q, k, v, out, table, i32([40]), n_queries=1, n_keys=40, k_scale=ks, v_scale=vs)
        outs.append(out)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and bool(torch.isfinite(outs[0].float()).all())
    assert float(outs[0].float().abs().max()) > 0


# ---------------------------------------------------------------------------
# the operators together
# ---------------------------------------------------------------------------

def decode_loop(stream=None, use_graph=False, steps=6):
    """Requests grow by a token a step: tables, append, selection, attention.  All outputs of all steps."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(4)
    R, H, G, D, page, width, keep = 3, 2, 4, 128, 16, 8, 4
    rows = torch.randn(steps, 2, 1, R, H, D, generator=gen, device=DEV).to(torch.bfloat16)
    qs = torch.randn(steps, R, H * G, D, generator=gen, device=DEV).to(torch.bfloat16)
    cache = km.Cache8.allocate(1, 40, page, H, D)
    prompt = torch.randn(2, R, 1, 90, H, D, generator=gen, device=DEV).to(torch.bfloat16)
    before, after = i32([0] * R), i32([90, 31, 64])
    table = torch.full((R, width), -1, dtype=torch.int32, device=DEV)
    free = torch.randperm(40, generator=gen, device=DEV).to(torch.int32)
    begin, end, base = i32([0]), i32([0]), i32([0] * (R + 1))
    slots = torch.zeros(200, dtype=torch.int64, device=DEV)
    km.page_tables(before, after, free, table, page_size=page, n_pool_pages=40, free_begin=begin, free_end=end,
                   token_base=base, slots=slots)
    km.append_paged8(prompt[0], prompt[1], cache.k, cache.v, cache.k_scale, cache.v_scale, table, chunk_tokens=after,
                     k_sum=cache.k_sum, k_sum_scale=cache.k_sum_scale)
    kv_row, q = torch.empty_like(rows[0]), torch.empty_like(qs[0])
    sel = torch.zeros((R, H, keep), dtype=torch.int32, device=DEV)
    count = torch.zeros((R, H), dtype=torch.int32, device=DEV)
    outs = [torch.zeros_like(q) for _ in range(2)]
    row_base = i32(range(R))
    calls = [
        km.prepare_page_tables(before, after, free, table, page_size=page, n_pool_pages=40, free_begin=begin,
                               free_end=end, token_base=base, slots=slots),
        km.prepare_append_paged8(kv_row[0], kv_row[1], cache.k, cache.v, cache.k_scale, cache.v_scale, table,
                                 n_tokens=1, tokens_before=before, row_base=row_base, k_sum=cache.k_sum,
                                 k_sum_scale=cache.k_sum_scale),
        km.prepare_select_pages(q, cache.k_sum[0], cache.k_sum_scale[0], table, after, sel, count, n_keys=width * page,
                                page_size=page),
        km.prepare_attend_paged(q, cache.k[0], cache.v[0], outs[0], table, after, n_queries=1, n_keys=width * page,
                                k_scale=cache.k_scale[0], v_scale=cache.v_scale[0], sel=sel, sel_count=count,
                                n_splits=2),
        km.prepare_attend_paged(q, cache.k[0], cache.v[0], outs[1], table, after, n_queries=1, n_keys=width * page,
                                k_scale=cache.k_scale[0], v_scale=cache.v_scale[0]),
    ]
    torch.cuda.synchronize()
    s = stream or torch.cuda.current_stream()

    def step():
        for c in calls:
            c.launch()

    graph = None
    if use_graph:
        # the capture itself runs nothing
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    got = []
    with torch.cuda.stream(s):
        for t in range(steps):
            before.copy_(after)
            after.add_(1)
            begin.copy_(end)
            kv_row.copy_(rows[t])
            q.copy_(qs[t])
            if graph is not None:
                graph.replay()
            else:
                step()
            s.synchronize()
            got.append([x.clone() for x in (table, slots, end, sel, count, outs[0], outs[1], cache.k_scale, cache.k_sum,
                                            cache.k.contiguous().view(torch.uint8))])
    torch.cuda.synchronize()
    return got


def test_decode_loop_on_a_stream_and_in_a_graph():
    """The same steps eagerly, on a stream of their own, and replayed from a graph, with eager work and waits
    between the replays: every step's outputs are the same bits."""
    eager = decode_loop()
    for other in (decode_loop(stream=torch.cuda.Stream()), decode_loop(use_graph=True)):
        for a, b in zip(eager, other):
            for x, y in zip(a, b):
                assert torch.equal(x, y)
    # the full attention of the last step differs from the selected pages' (pages were left out)
    assert not torch.equal(eager[-1][5], eager[-1][6])


def test_example_answers_from_recalled_chunks():
    """The example's steps from its graph equal the eager ones, and its last answer token the plain form over
    the cache that it leaves."""
    from examples.answer_from_recall import answer

    kw = dict(chunks=3, tokens=64, layers=2, question=20, steps=3, keep=6, seed=9)
    torch.manual_seed(1)
    out_q, answers, r = answer(**kw)
    torch.manual_seed(1)
    out_q2, answers2, _ = answer(graph=False, **kw)
    assert torch.equal(out_q, out_q2) and torch.equal(answers, answers2)
    n = int(r.tokens)
    assert n == 3 * 64 + 20 + 3 and int(r.count.min()) == 6
    gen = torch.Generator(device=DEV)
    gen.manual_seed(9)
    # the last layer's query of the last step, drawn again in the example's order
    q = last_query(gen, kw)
    bytes_ = r.cache.k[1].contiguous().view(torch.uint8).cpu().numpy()
    v_bytes = r.cache.v[1].contiguous().view(torch.uint8).cpu().numpy()
    ks, vs = r.cache.k_scale[1].cpu().double().numpy(), r.cache.v_scale[1].cpu().double().numpy()
    k, v = ref.decode(bytes_) * ks[:, None, :, None], ref.decode(v_bytes) * vs[:, None, :, None]
    table = r.table.cpu().numpy()
    sel = [[int(x) for x in r.sel[0, h].cpu() if x >= 0] for h in range(8)]
    k_sum, k_sum_scale = r.cache.k_sum[1].cpu().numpy(), r.cache.k_sum_scale[1].cpu().double().numpy()
    qv = q.double().cpu().numpy()
    assert sel == ref.select(qv, k_sum, k_sum_scale, table, [n], 16, 6, 1, 2)
    a = (table, [n], [1], [0], 16, 128 ** -0.5, True, 0, sel)
    want, _ = ref.attend(qv, k, v, *a)
    size, _ = ref.attend(qv, k, np.abs(v), *a)
    got = answers[-1, 1].double().cpu().numpy()
    assert (np.abs(got - want) <= BOUND * size).all()


def last_query(gen, kw):
    def rows(*shape):
        return torch.randn(shape, generator=gen, device=DEV).to(torch.bfloat16)

    c, n, layers = kw["chunks"], kw["tokens"], kw["layers"]
    rows(c, layers, n, 8, 128), rows(c, layers, n, 8, 128)
    rows(2, c, layers, 8, n, 16), rows(2, c, layers, 8, 16, 128)
    rows(2, 1, layers, kw["question"], 8, 128)
    for _ in range(layers):
        rows(kw["question"], 64, 128)
    for _ in range(kw["steps"]):
        rows(2, 1, layers, 1, 8, 128)
        q = rows(layers, 1, 64, 128)
    return q[-1]


def test_calls_on_a_given_stream():
    """Calls handed a stream (an object or a raw handle) run there, after what that stream holds already, and a
    workspace of their own outlives the call."""
    s = attend_case(dict(kv=[3000, 700], H=2, G=4))
    table, kv = i32(s["table"]), i32(s["kv"])
    want = torch.zeros_like(s["q"])
    km.attend_paged(s["q"], s["kt"], s["vt"], want, table, kv, n_queries=1, n_keys=3000, **s["scales"])
    torch.cuda.synchronize()
    for raw in (False, True):
        side = torch.cuda.Stream()
        q = torch.zeros_like(s["q"])
        out = torch.zeros_like(s["q"])
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(2_000_000)
            q.copy_(s["q"])
        km.attend_paged(q, s["kt"], s["vt"], out, table, kv, n_queries=1, n_keys=3000, n_splits=4,
                        stream=side.cuda_stream if raw else side, **s["scales"])
        # memory that the current stream takes meanwhile is not the call's workspace
        noise = [torch.full((1 << 20,), float("nan"), device=DEV) for _ in range(4)]
        side.synchronize()
        assert len(noise) == 4
        assert float((out.float() - want.float()).abs().max()) <= 2.0 ** -6


@pytest.mark.parametrize("raw", ["object", "raw", "null"])
def test_own_workspace_is_memory_of_the_given_stream(raw, monkeypatch):
    """Memory of another stream may still be read there when this call writes it."""
    s = attend_case(dict(kv=[3000, 700], H=2, G=4))
    table, kv, out = i32(s["table"]), i32(s["kv"]), torch.zeros_like(s["q"])
    side = torch.cuda.default_stream() if raw == "null" else torch.cuda.Stream()
    torch.cuda.synchronize()
    taken, empty = [], torch.empty

    def seen(*a, **kw):
        taken.append(torch.cuda.current_stream().cuda_stream)
        return empty(*a, **kw)

    monkeypatch.setattr(torch, "empty", seen)
    km.attend_paged(s["q"], s["kt"], s["vt"], out, table, kv, n_queries=1, n_keys=3000, n_splits=4,
                    stream=side if raw == "object" else side.cuda_stream, **s["scales"])
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert taken == [side.cuda_stream]
    check_attend(out, None, s, 128 ** -0.5)


def test_calls_take_any_object_that_has_a_stream():
    """As the package's other calls do: what has a cuda_stream."""
    s = attend_case(dict(kv=[3000, 700], H=2, G=4))

    class Handle:
        pass

    out, side, handle = torch.zeros_like(s["q"]), torch.cuda.Stream(), Handle()
    handle.cuda_stream = side.cuda_stream
    torch.cuda.synchronize()
    km.attend_paged(s["q"], s["kt"], s["vt"], out, i32(s["table"]), i32(s["kv"]), n_queries=1, n_keys=3000, n_splits=4,
                    stream=handle, **s["scales"])
    torch.cuda.synchronize()
    check_attend(out, None, s, 128 ** -0.5)


@pytest.mark.parametrize("cache", ["e4m3", "bf16"])
@pytest.mark.parametrize("queries", [1, 3, 40])
def test_a_query_that_is_not_finite_stays_in_its_row(cache, queries):
    s = attend_case(dict(kv=[150], nq=[queries], H=2, G=4, cache=cache))
    clean, out = torch.zeros_like(s["q"]), torch.zeros_like(s["q"])
    table, kv = i32(s["table"]), i32(s["kv"])
    km.attend_paged(s["q"], s["kt"], s["vt"], clean, table, kv, n_queries=queries, n_keys=150, **s["scales"])
    q = s["q"].clone()
    q[queries // 2, 5, 9] = float("nan")
    km.attend_paged(q, s["kt"], s["vt"], out, table, kv, n_queries=queries, n_keys=150, **s["scales"])
    torch.cuda.synchronize()
    hit = torch.zeros(s["q"].shape[:2], dtype=torch.bool, device=DEV)
    hit[queries // 2, 5] = True
    assert torch.isnan(out[hit].float()).all()
    assert torch.equal(out[~hit], clean[~hit])


def test_parts_of_a_context_join_by_lse():
    """Attention over two halves of the pages, joined by their lse, is the attention over all of them."""
    s = attend_case(dict(kv=[640, 640], H=2, G=4, page=32))
    table, n = i32(s["table"]), 640
    outs, lses = [], []
    for a, b in ((0, 20), (0, 7), (7, 20)):
        out, lse = torch.zeros_like(s["q"]), torch.zeros(s["q"].shape[:2], device=DEV)
        km.attend_paged(s["q"], s["kt"], s["vt"], out, table[:, a:b], i32([(b - a) * 32] * 2), n_queries=1,
                        n_keys=(b - a) * 32, causal=False, lse=lse, **s["scales"])
        outs.append(out.double())
        lses.append(lse.double())
    torch.cuda.synchronize()
    w = torch.softmax(torch.stack(lses[1:]), 0)[..., None]
    joined = w[0] * outs[1] + w[1] * outs[2]
    size, _ = ref.attend(s["qv"], s["k"], np.abs(s["v"]), s["table"], s["kv"], s["nq"], s["base"], 32, 128 ** -0.5,
                         False)
    # each side within BOUND of the exact one
    assert (np.abs((joined - outs[0]).cpu().numpy()) <= 2 * BOUND * size).all()
    assert float((torch.logsumexp(torch.stack(lses[1:]), 0) - lses[0]).abs().max()) <= 2.0 ** -10
