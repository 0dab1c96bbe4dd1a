"""The latent-cache operators on the GPU against plain 64-bit forms (latent_ref).

Bounds, with u = 2^-8 the largest relative error of a rounding to bf16:
  rotated element   the sum of two products of fp32 numbers, rounded once.  The angle is
                    off by less than 2^-20 (fp64 product, one fp32 rounding of the reduced
                    revolutions), the hardware's sine and cosine by less than 2^-19:
                    u |ref| + 2^-18 (|x| + |y|)
  product           n_in products summed in fp32: u |ref| + (n_in + 2) 2^-24 sum |x w|
  attention         a weight is rounded to bf16 and their sum taken of the rounded ones: off
                    by at most u of the spread sum p |v - out| <= 2 sum p |v|; the output is
                    rounded once.  A score, D products summed in fp32, is off by
                    e = (D + 8) 2^-24 max sum |q_j k_j| scale, which moves p / sum p by 2 e at
                    most; exponentials, sums and the joining of parts by less than 2^-18:
                    (3 u + 4 e + 2^-18) sum p |v|, and lse 2 e + 2^-18 (1 + |lse|).
"""

from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2606_23581_amd as km
from tests import latent_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"
U = 2.0 ** -8


def i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device=DEV)


def bf16(x):
    """float64 numpy -> (bf16 device tensor, its values)."""
    t = torch.tensor(np.asarray(x, dtype=np.float32)).to(torch.bfloat16)
    return t.to(DEV), t.double().numpy()


def values(t):
    return t.double().cpu().numpy()


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy()


def table_for(rng, lengths, page, width=None, spare=3):
    need = [-(-n // page) for n in lengths]
    pool = sum(need) + spare
    order = rng.permutation(pool)
    t = np.full((len(lengths), max([1, width or 0] + need)), -1, dtype=np.int32)
    at = 0
    for r, n in enumerate(need):
        t[r, :n] = order[at:at + n]
        at += n
    return t, pool


# ---------------------------------------------------------------------------
# rotated append
# ---------------------------------------------------------------------------

APPEND_CASES = {
    "one_token": dict(before=[0], tokens=[1]),
    "latent_step": dict(before=[15, 16, 17, 0, 500], tokens=[1] * 5, H=1, D=576, rope=(512, 64), v=None, HQ=16,
                        pairing="interleaved"),
    "latent_neox": dict(before=[3, 100], tokens=[40, 17], H=1, D=576, rope=(512, 64), v=None, HQ=5),
    "prompt": dict(before=[0, 33], tokens=[70, 41], H=2, D=128, HQ=7),
    "odd_heads": dict(before=[5], tokens=[19], H=3, D=64, rope=(0, 64), HQ=9, pairing="interleaved"),
    "partial_band": dict(before=[9, 0], tokens=[33, 2], H=2, D=128, rope=(32, 32), HQ=4),
    "narrow_band": dict(before=[9, 0], tokens=[33, 2], H=2, D=72, rope=(40, 16), HQ=4),
    "narrow_interleaved": dict(before=[9, 0], tokens=[33, 2], H=1, D=40, rope=(16, 8), HQ=3, pairing="interleaved"),
    "sections": dict(before=[4, 8], tokens=[20, 31], H=2, D=128, sections=(24, 20, 20), HQ=4),
    "sections_interleaved": dict(before=[4], tokens=[20], H=1, D=64, rope=(0, 64), sections=(16, 8, 8), HQ=4,
                                 order="interleaved", pairing="interleaved"),
    "positions": dict(before=[4, 8], tokens=[20, 31], H=2, D=128, positions=True, HQ=4),
    "far": dict(before=[2000000000], tokens=[7], H=1, D=128, positions=True, far=True, HQ=2),
    "linear": dict(before=[4000], tokens=[20], H=2, D=128, scaling=dict(kind="linear", factor=4.0)),
    "turns": dict(before=[4000], tokens=[20], H=2, D=128, HQ=3,
                  scaling=dict(kind="turns", factor=8.0, original_tokens=8192, low_turns=1.0, high_turns=4.0)),
    "pairs": dict(before=[40000], tokens=[20], H=1, D=576, rope=(512, 64), v=None, HQ=4, pairing="interleaved",
                  scaling=dict(kind="pairs", factor=40.0, original_tokens=4096, amplitude=1.3689)),
    "pairs_steep": dict(before=[40], tokens=[20], H=1, D=64, rope=(0, 64), HQ=4,
                        scaling=dict(kind="pairs", factor=4.0, original_tokens=8, low_turns=5.0, high_turns=6.0,
                                     amplitude=-0.5)),
    "layers_unpacked": dict(before=[5, 0, 30], tokens=[9, 16, 1], H=2, D=64, rope=(0, 64), L=3, packed=False, HQ=2),
    "layers_packed": dict(before=[5, 0, 30], tokens=[9, 16, 1], H=2, D=64, rope=(0, 64), L=3, HQ=2),
    "zero_tokens": dict(before=[5, 9], tokens=[0, 3]),
    "no_before": dict(before=None, tokens=[33, 5], HQ=2),
    "odd_page": dict(before=[5, 13], tokens=[30, 9], page=7),
    "page_of_one": dict(before=[1], tokens=[5], page=1),
    "bad_page": dict(before=[5, 13], tokens=[60, 30], bad=[(0, 1), (1, 2)], HQ=3),
    "outgrow": dict(before=[5, 13], tokens=[60, 30], width=2, HQ=3),
    "values_wider": dict(before=[5], tokens=[20], H=2, D=64, rope=(0, 64), v=(3, 136)),
    "in_place": dict(before=[5, 700], tokens=[20, 40], HQ=5, in_place=True),
    "many": dict(before=list(range(0, 300, 3)), tokens=[(7 * c) % 5 for c in range(100)], H=1, D=64, rope=(0, 64), HQ=2),
}


@pytest.mark.parametrize("name", sorted(APPEND_CASES))
def test_append_rotated(name):
    c = dict(page=16, H=2, D=128, HQ=0, v="same", L=1, packed=True, pairing="neox", scaling=None, bad=(), positions=False)
    c.update(APPEND_CASES[name])
    rng = np.random.default_rng(5)
    tokens, page, H, D, L = c["tokens"], c["page"], c["H"], c["D"], c["L"]
    C = len(tokens)
    before = c["before"] or [0] * C
    held = [b % 1000 for b in before] if c.get("far") else before
    off, rd = c.get("rope", (0, D))
    VH, VD = (H, D) if c["v"] == "same" else c["v"] or (0, 0)
    lengths = [b + t for b, t in zip(held, tokens)]
    table, pool = table_for(rng, [min(n, c.get("width", 10 ** 9) * page) for n in lengths], page, width=c.get("width"))
    for r, j in c["bad"]:
        table[r, j] = pool + 3 if r else -7
    n = max(tokens)
    starts = [sum(tokens[:r]) + 2 for r in range(C)]
    shape = (L, sum(tokens) + 5) if c["packed"] else (C, L, n)
    k, k64 = bf16(rng.standard_normal((*shape, H, D)))
    v, v64 = bf16(rng.standard_normal((*shape, max(VH, 1), max(VD, 8))))
    q, q64 = bf16(rng.standard_normal((*shape, max(c["HQ"], 1), rd + 16)))
    q_in = q[..., 8:8 + rd]
    q_out = q_in if c.get("in_place") else torch.full((*q.shape[:-1], rd + 8), -7.0, dtype=torch.bfloat16, device=DEV)[..., 8:]
    kc, kc64 = bf16(rng.standard_normal((L, pool, page, H, D)))
    vc, vc64 = bf16(rng.standard_normal((L, pool, page, max(VH, 1), max(VD, 8))))
    sections = c.get("sections")
    pos = None
    if sections or c["positions"]:
        lead = (shape[1],) if c["packed"] else (C, n)
        hi = (1 << 31) - 1 if c.get("far") else 40000
        pos = rng.integers(-hi if c.get("far") else 0, hi, size=(*lead, 3 if sections else 1))
    sc = c["scaling"]
    rope = km.RopeSpec(theta=1e6, rope_dim=rd, rope_offset=off, pairing=c["pairing"], sections=sections,
                       section_order=c.get("order", "blocked"))
    status = i32([0])
    km.append_rotated(k, v if VH else None, kc, vc if VH else None, i32(table), rope=rope,
                      scaling=km.RopeScaling(**sc) if sc else None, positions=None if pos is None else i32(pos),
                      n_tokens=n, tokens_before=i32(held) if c["before"] else None, chunk_tokens=i32(tokens),
                      row_base=i32(starts) if c["packed"] else None, q=q_in if c["HQ"] else None,
                      q_out=q_out if c["HQ"] else None, status=status)
    torch.cuda.synchronize()

    sc = sc or dict(kind="none")
    f = ref.frequencies(1e6, rd, sc["kind"], sc.get("factor", 1.0), sc.get("original_tokens", 0), sc.get("low_turns", 1.0),
                        sc.get("high_turns", 32.0))
    coord = np.zeros(rd // 2, dtype=int)
    if sections:
        if c.get("order") == "interleaved":
            left, j = list(sections), 0
            while j < rd // 2:
                for x in range(3):
                    if left[x] and j < rd // 2:
                        coord[j], j, left[x] = x, j + 1, left[x] - 1
        else:
            coord = np.repeat([0, 1, 2], sections)
    amp = sc.get("amplitude", 1.0)
    want_k, tol_k, want_v = kc64.copy(), np.zeros_like(kc64), vc64.copy()
    got_q, seen_q, flags = values(q_out), np.zeros(q_out.shape[:-2], dtype=bool), 0
    for ch in range(C):
        for i in range(tokens[ch]):
            tok = held[ch] + i
            at = (slice(None), starts[ch] + i) if c["packed"] else (ch, slice(None), i)
            p = pos[at[1:] if c["packed"] else (ch, i)][coord] if pos is not None else np.full(rd // 2, tok)
            angle = np.array([float(np.longdouble(x) * np.longdouble(y) % (2 * np.longdouble(np.pi))) for x, y in zip(p, f)])
            if c["HQ"]:
                r, size = ref.rotate(q64[at][..., 8:8 + rd], angle, c["pairing"], amp)
                np.testing.assert_array_less(np.abs(got_q[at] - r), U * np.abs(r) + 2.0 ** -18 * size + 1e-30)
                seen_q[at] = True
            if tok // page >= table.shape[1]:
                flags |= km.STATUS_BAD_LENGTH
                continue
            pg = table[ch, tok // page]
            if not 0 <= pg < pool:
                flags |= km.STATUS_BAD_PAGE
                continue
            want_k[:, pg, tok % page] = k64[at]
            r, size = ref.rotate(k64[at][..., off:off + rd], angle, c["pairing"], amp)
            want_k[:, pg, tok % page, :, off:off + rd] = r
            tol_k[:, pg, tok % page, :, off:off + rd] = U * np.abs(r) + 2.0 ** -18 * size
            want_v[:, pg, tok % page] = v64[at]
    err = np.abs(values(kc) - want_k)
    assert (err <= tol_k).all(), float((err - tol_k).max())
    np.testing.assert_array_equal(values(vc), want_v if VH else vc64)
    assert int(status) == flags
    # queries' other columns and rows keep their bits
    if c["HQ"] and not c.get("in_place"):
        assert (got_q[~seen_q] == -7).all()
    if c.get("in_place"):
        now = values(q)
        np.testing.assert_array_equal(now[..., :8], q64[..., :8])
        np.testing.assert_array_equal(now[..., 8 + rd:], q64[..., 8 + rd:])
        np.testing.assert_array_equal(now[~seen_q], q64[~seen_q])


def test_append_rotated_agrees_with_rehydrate():
    """Rows appended at positions p and rows rehydrated there are the same bits: one rotation."""
    torch.manual_seed(0)
    n, D, page = 40, 576, 16
    rows = torch.randn(1, 1, n, 1, D, device=DEV).to(torch.bfloat16)
    rope = km.RopeSpec(theta=1e4, rope_dim=64, rope_offset=512, pairing="interleaved")
    table = i32([[4, 0, 2]])
    a, b = (torch.zeros(1, 5 * page, 1, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    km.rehydrate(rows, a, rope=rope, chunk_pos=i32([[0, 0, 0]]), page_table=table, page_size=page, n_pool_pages=5)
    km.append_rotated(rows, None, b.view(1, 5, page, 1, D), None, table, rope=rope)
    assert torch.equal(a, b)


def test_append_rotated_fused_rows():
    """Queries, keys and values as columns of one tensor, queries rotated in place."""
    torch.manual_seed(1)
    n, HQ, H, D, page = 37, 8, 2, 64, 16
    x = torch.randn(1, n, (HQ + 2 * H), D, device=DEV).to(torch.bfloat16)
    before = x.clone()
    pool = torch.zeros(1, 4, page, 2, H, D, dtype=torch.bfloat16, device=DEV)
    q, k, v = x[:, :, :HQ], x[:, :, HQ:HQ + H], x[:, :, HQ + H:]
    km.append_rotated(k, v, pool[:, :, :, 0], pool[:, :, :, 1], i32([[3, 1, 0]]), rope=km.RopeSpec(theta=1e4, rope_dim=D),
                      n_tokens=n, row_base=i32([0]), q=q, q_out=q)
    assert torch.equal(x[:, :, HQ:], before[:, :, HQ:])
    f = ref.frequencies(1e4, D)
    got, want = values(q)[0], values(before)[0]
    for i in range(n):
        r, size = ref.rotate(want[i, :HQ], i * f, "neox")
        assert (np.abs(got[i] - r) <= U * np.abs(r) + 2.0 ** -18 * size).all()
    np.testing.assert_array_equal(bits(pool[0, 3, :, 1]), bits(before[0, :16, HQ + H:]))


# ---------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------

def product_bound(x, w):
    y = x @ w
    return y, U * np.abs(y) + (x.shape[-1] + 2) * 2.0 ** -24 * (np.abs(x) @ np.abs(w)) + 1e-30


@pytest.mark.parametrize("w_rows", [True, False])
@pytest.mark.parametrize("rows,heads,n_in,n_out", [(1, 1, 64, 64), (1, 16, 128, 512), (3, 5, 512, 128), (33, 2, 192, 320),
                                                   (64, 3, 128, 128), (65, 3, 64, 192), (127, 1, 256, 64),
                                                   (129, 4, 128, 512), (300, 2, 576, 448), (1000, 3, 512, 128),
                                                   (300, 256, 64, 256), (515, 90, 192, 512)])
def test_project_heads(rows, heads, n_in, n_out, w_rows):
    rng = np.random.default_rng(rows)
    x, x64 = bf16(rng.standard_normal((rows, heads, n_in)))
    w, w64 = bf16(rng.standard_normal((heads, n_in, n_out)))
    if not w_rows:
        w = w.transpose(1, 2).contiguous().transpose(1, 2)
    out = torch.full((rows + 1, heads, n_out), 9.0, dtype=torch.bfloat16, device=DEV)
    km.project_heads(x, w, out[:rows])
    for h in range(heads):
        y, tol = product_bound(x64[:, h], w64[h])
        err = np.abs(values(out[:rows, h]) - y)
        assert (err <= tol).all(), (h, float((err / tol).max()))
    assert (out[rows] == 9.0).all()


@pytest.mark.parametrize("rows", [5, 200])
def test_project_heads_views(rows):
    """Bands of wider rows in and out, x or W shared by the heads, transposed outputs."""
    rng = np.random.default_rng(0)
    q, q64 = bf16(rng.standard_normal((rows, 4, 192)))
    w, w64 = bf16(rng.standard_normal((4, 192, 256)))
    out = torch.full((4, rows, 264), 3.0, dtype=torch.bfloat16, device=DEV)
    km.project_heads(q[..., 64:], w[:, :128, :192], out.transpose(0, 1)[..., 8:200])
    km.project_heads(q[:, :1, 64:].expand(-1, 4, -1), w[:, 64:, 128:192], out.transpose(0, 1)[..., 200:])
    for h in range(4):
        y, tol = product_bound(q64[:, h, 64:], w64[h, :128, :192])
        assert (np.abs(values(out[h, :, 8:200]) - y) <= tol).all()
        y, tol = product_bound(q64[:, 0, 64:], w64[h, 64:, 128:192])
        assert (np.abs(values(out[h, :, 200:]) - y) <= tol).all()
    assert (out[:, :, :8] == 3.0).all()
    out2 = torch.zeros(rows, 4, 192, dtype=torch.bfloat16, device=DEV)
    km.project_heads(q[..., :128], w[1:2, :128, :192].expand(4, -1, -1), out2)
    y, tol = product_bound(q64[:, 3, :128], w64[1, :128, :192])
    assert (np.abs(values(out2[:, 3]) - y) <= tol).all()


def test_project_heads_not_finite_stays_in_its_row():
    x = torch.ones(70, 2, 128, dtype=torch.bfloat16, device=DEV)
    w = torch.ones(2, 128, 64, dtype=torch.bfloat16, device=DEV)
    x[3, 1, 5], x[69, 0, 0] = float("nan"), float("inf")
    out = torch.zeros(70, 2, 64, dtype=torch.bfloat16, device=DEV)
    km.project_heads(x, w, out)
    want = torch.full_like(out, 128.0)
    want[3, 1], want[69, 0] = float("nan"), float("inf")
    assert torch.equal(torch.nan_to_num(out.float(), 7.0), torch.nan_to_num(want.float(), 7.0))


@pytest.mark.parametrize("w_rows", [True, False])
@pytest.mark.parametrize("lengths,page,heads,n_in,n_out", [([1], 16, 1, 256, 64), ([5, 0, 17, 64], 16, 3, 512, 128),
                                                           ([200, 33], 7, 2, 512, 192), ([300, 129, 128], 64, 4, 256, 256),
                                                           ([20] * 40, 16, 2, 64, 128),
                                                           ([257, 31, 300] * 16, 16, 6, 64, 256)])
def test_expand_latent(lengths, page, heads, n_in, n_out, w_rows):
    rng = np.random.default_rng(2)
    table, pool = table_for(rng, lengths, page)
    cache, c64 = bf16(rng.standard_normal((pool, page, n_in + 64)))
    w, w64 = bf16(rng.standard_normal((heads, n_in, n_out)))
    if not w_rows:
        w = w.transpose(1, 2).contiguous().transpose(1, 2)
    bad = len(lengths) > 1 and lengths[0] > page
    if bad:
        table[0, 1] = pool
    base = [sum(lengths[:r]) + 3 * r for r in range(len(lengths))]
    out = torch.full((sum(lengths) + 3 * len(lengths), heads, n_out), 5.0, dtype=torch.bfloat16, device=DEV)
    status = i32([0])
    km.expand_latent(cache, w, out, i32(table), i32(lengths), n_keys=max(lengths), row_base=i32(base), status=status)
    got, left = values(out), np.ones(out.shape[0], dtype=bool)
    for r, n in enumerate(lengths):
        x, ok = ref.gather(c64, table[r], n, page)
        for t in np.flatnonzero(ok):
            left[base[r] + t] = False
        for h in range(heads):
            y, tol = product_bound(x[:, :n_in], w64[h])
            assert (np.abs(got[base[r]:base[r] + n, h] - y) <= tol)[ok].all()
    assert (got[left] == 5.0).all()
    assert int(status) == (km.STATUS_BAD_PAGE if bad else 0)
    # without a row base: rows r * n_keys + t
    out2 = torch.full((len(lengths) * max(lengths), heads, n_out), 5.0, dtype=torch.bfloat16, device=DEV)
    km.expand_latent(cache, w, out2, i32(table), i32(lengths), n_keys=max(lengths))
    for r, n in enumerate(lengths):
        assert torch.equal(out2[r * max(lengths):r * max(lengths) + n], out[base[r]:base[r] + n])
        assert (out2[r * max(lengths) + n:(r + 1) * max(lengths)] == 5.0).all()


# Shapes that are taken in tiles of 256 rows and columns (test_latent_abi.py asserts that they are).
PROJECT_256 = [(515, 85, 192, 512), (257, 97, 128, 256), (300, 64, 512, 512)]          # rows, heads, in, out
EXPAND_256 = [([257, 31, 300] * 16, 16, 4, 192, 256), ([300, 0, 256, 255] * 12, 64, 2, 512, 512),  # lengths, page, heads, in, out
              ([1100, 1300], 7, 20, 320, 256)]


@pytest.mark.parametrize("w_rows", [True, False])
@pytest.mark.parametrize("rows,heads,n_in,n_out", PROJECT_256)
def test_project_heads_in_tiles_of_256(rows, heads, n_in, n_out, w_rows):
    test_project_heads(rows, heads, n_in, n_out, w_rows)


@pytest.mark.parametrize("w_rows", [True, False])
@pytest.mark.parametrize("lengths,page,heads,n_in,n_out", EXPAND_256)
def test_expand_latent_in_tiles_of_256(lengths, page, heads, n_in, n_out, w_rows):
    """Ragged requests, and one with a page outside the pool."""
    test_expand_latent(lengths, page, heads, n_in, n_out, w_rows)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

ATTEND_CASES = {
    "one_key": dict(kv=[1], nq=[1]),
    "short": dict(kv=[5, 16, 17, 31, 33], nq=[1] * 5),
    "unit_edges": dict(kv=[127, 128, 129, 256, 300], nq=[1] * 5, H=4),
    "no_keys": dict(kv=[0, 20, 0], nq=[1, 1, 3]),
    "no_queries": dict(kv=[30, 20], nq=[0, 2]),
    "one_head": dict(kv=[40, 100], nq=[1, 2], H=1),
    "odd_heads": dict(kv=[40, 100], nq=[3, 1], H=5),
    "rows_16": dict(kv=[70, 200], nq=[1, 1], H=16),
    "rows_17": dict(kv=[70, 200], nq=[1, 1], H=17),
    "rows_33": dict(kv=[170, 200], nq=[3, 2], H=11),
    "rows_64": dict(kv=[170, 200], nq=[4, 2], H=16),
    "rows_65": dict(kv=[170, 200], nq=[5, 2], H=13),
    "rows_128": dict(kv=[170, 250], nq=[1, 1], H=128),
    "rows_129": dict(kv=[170, 60], nq=[3, 1], H=43),
    "chunk": dict(kv=[100, 300], nq=[40, 30], H=8),
    "whole_prompt": dict(kv=[50, 140], nq=[50, 140], H=2),
    "more_queries_than_keys": dict(kv=[10, 3, 70], nq=[16, 12, 70], H=3),
    "not_causal": dict(kv=[70, 33], nq=[5, 12], causal=False, H=4),
    "window_1": dict(kv=[70, 200], nq=[1, 4], window=1, H=4),
    "window": dict(kv=[170, 300, 20], nq=[1, 30, 2], window=50, H=4),
    "window_decode": dict(kv=[500, 300, 20], nq=[1, 1, 1], window=100, H=16),
    "window_past_all": dict(kv=[70], nq=[40], window=1 << 40, H=4),
    "page_48": dict(kv=[170, 49], nq=[2, 1], page=48, H=4),
    "page_64": dict(kv=[170, 300], nq=[2, 7], page=64, H=4),
    "bad_page": dict(kv=[170, 100, 40], nq=[1, 20, 3], bad=[(0, 2), (1, 0), (1, 6)], H=4),
    "all_pages_bad": dict(kv=[20, 40], nq=[2, 2], bad=[(0, 0), (0, 1)], H=4),
    "negative_scale": dict(kv=[70, 33], nq=[2, 1], scale=-0.05, H=4),
    "zero_scale": dict(kv=[70, 33], nq=[2, 1], scale=0.0, H=4),
    "large_scores": dict(kv=[200], nq=[3], scale=1.0, H=4),
    "long": dict(kv=[3000, 1500], nq=[1, 1], H=16),
    "long_queries": dict(kv=[3000, 700], nq=[2, 3], H=16),
    "long_wide": dict(kv=[1200, 700], nq=[1, 2], H=40),
}


def attend(form, c, parts=0, D=None, seed=7, poison=None):
    """One call of a form: (got out, got lse, wanted out, size, wanted lse, most, base rows)."""
    c = dict(dict(H=16, page=16, causal=True, window=0, scale=None, bad=()), **c)
    rng = np.random.default_rng(seed)
    H, page, kv, nq = c["H"], c["page"], c["kv"], c["nq"]
    D = D or (512 if form == "latent" else 128)
    table, pool = table_for(rng, kv, page, -(-c.get("most", (0, 0))[1] // page))
    for r, j in c["bad"]:
        table[r, j] = -1 if j % 2 else pool + 2
    width = (D if form == "latent" else 512) + 64
    rows, rows64 = bf16(rng.standard_normal((pool, page, width)))
    used = np.zeros((pool, page), dtype=bool)
    for r, n in enumerate(kv):
        for t in range(n):
            if 0 <= table[r, t // page] < pool:
                used[table[r, t // page], t % page] = True
    rows[torch.tensor(~used, device=DEV)] = float("nan")
    base = [sum(nq[:r]) + r for r in range(len(nq))]
    n_rows = sum(nq) + len(nq) + 1
    q, q64 = bf16(rng.standard_normal((n_rows, H, D + 64)) * (0.5 if form == "latent" else 1.0))
    scale = c["scale"] if c["scale"] is not None else 192 ** -0.5
    out = torch.full((n_rows, H, D), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((n_rows, H), 7.0, device=DEV)
    status = i32([0])
    most_q, most_kv = c.get("most", (max(nq), max(kv)))
    kw = dict(n_queries=most_q, n_keys=most_kv, scale=scale, q_base=i32(base), q_tokens=i32(nq), causal=c["causal"],
              window=c["window"], lse=lse, n_parts=parts, status=status)
    if form == "latent":
        if poison is not None:
            poison(rows, rows64, table)
        km.attend_latent(q, rows, out, i32(table), i32(kv), **kw)
    else:
        kv_base = [sum(kv[:r]) + 2 * r for r in range(len(kv))]
        ex, ex64 = bf16(rng.standard_normal((sum(kv) + 2 * len(kv) + 2, H, 2 * D)))
        free = np.ones(ex.shape[0], dtype=bool)
        for r, n in enumerate(kv):
            free[kv_base[r]:kv_base[r] + n] = False
        ex[torch.tensor(free, device=DEV)] = float("nan")
        if poison is not None:
            poison(ex, ex64, kv_base)
        km.attend_expanded(q, ex[..., :D], ex[..., D:], rows[..., -64:], out, i32(table), i32(kv), kv_base=i32(kv_base), **kw)
    torch.cuda.synchronize()
    want, size = np.full((n_rows, H, D), 7.0), np.zeros((n_rows, H, D))
    want_lse, most = np.full((n_rows, H), 7.0), 0.0
    for r, n in enumerate(kv):
        x, ok = ref.gather(rows64, table[r], n, page)
        seen = ref.seen_keys(n, nq[r], c["causal"], min(c["window"], 1 << 30), ok)
        if form == "latent":
            k, v = x[None], x[None, :, :D]
        else:
            e = ex64[kv_base[r]:kv_base[r] + n].transpose(1, 0, 2)
            k = np.concatenate([e[..., :D], np.broadcast_to(x[None, :, -64:], (H, n, 64))], -1)
            v = e[..., D:]
        at = slice(base[r], base[r] + nq[r])
        want[at], size[at], want_lse[at], m = ref.attend_rows(q64[at], k, v, seen, scale)
        most = max(most, m)
    bad = any(b[0] < len(kv) and b[1] * page < kv[b[0]] for b in c["bad"])
    assert int(status) == (km.STATUS_BAD_PAGE if bad else 0)
    return values(out), values(lse), want, size, want_lse, most * (D + 64 + 8) * 2.0 ** -24


def check(got, got_lse, want, size, want_lse, e):
    tol = (3 * U + 4 * e + 2.0 ** -18) * size
    err = np.abs(got - want)
    assert (err <= tol).all(), float((err / np.maximum(tol, 1e-30)).max())
    np.testing.assert_array_equal(np.isinf(got_lse), np.isinf(want_lse))
    fin = np.isfinite(want_lse)
    assert (np.abs(got_lse - want_lse)[fin] <= 2 * e + 2.0 ** -18 * (1 + np.abs(want_lse[fin]))).all()


@pytest.mark.parametrize("form", ["latent", "expanded"])
@pytest.mark.parametrize("name", sorted(ATTEND_CASES))
def test_attend(form, name):
    check(*attend(form, ATTEND_CASES[name]))


@pytest.mark.parametrize("form,D", [("latent", 256), ("expanded", 64)])
@pytest.mark.parametrize("name", ["short", "rows_17", "rows_33", "rows_65", "chunk", "window", "bad_page", "long", "no_keys"])
def test_attend_smaller_columns(form, D, name):
    check(*attend(form, ATTEND_CASES[name], D=D))


@pytest.mark.parametrize("form", ["latent", "expanded"])
@pytest.mark.parametrize("parts", [1, 2, 7, 64, 1000])
@pytest.mark.parametrize("name", ["no_keys", "unit_edges", "rows_17", "rows_33", "rows_65", "rows_129", "chunk", "window",
                                  "more_queries_than_keys", "bad_page", "long_wide", "no_queries"])
def test_attend_divided(form, parts, name):
    check(*attend(form, ATTEND_CASES[name], parts=parts))


POISON_CASES = {
    "causal": dict(kv=[60, 40], nq=[7, 3], H=4),
    "causal_rows": dict(kv=[300, 200], nq=[33, 40], H=5),
    "window": dict(kv=[300, 200], nq=[20, 11], H=4, window=30),
    "prompt": dict(kv=[150], nq=[150], H=2),
}


# More requests than a wave has lanes, empty ones among them; lengths that leave most of the sizes' room unused.
MANY_CASES = {
    "one_query": dict(kv=[(37 * r) % 90 for r in range(150)] + [900], nq=[1] * 151, H=4),
    "blocks": dict(kv=[(53 * r) % 70 for r in range(70)] + [400], nq=[(11 * r) % 26 for r in range(70)] + [150], H=8),
    "last_alone": dict(kv=[0] * 129 + [800], nq=[0] * 129 + [3], H=2),
    "first_alone": dict(kv=[800] + [0] * 129, nq=[3] + [0] * 129, H=2),
    "all_empty": dict(kv=[0] * 70 + [0], nq=[0] * 70 + [0], H=2, most=(4, 600)),
    "whole_tasks": dict(kv=[600, 0, 1, 300] + [(7 * r) % 4 for r in range(2044)], nq=[3, 1, 1, 0] + [1] * 2044, H=2),
}


@pytest.mark.parametrize("form", ["latent", "expanded"])
@pytest.mark.parametrize("parts", [0, 1, 9, 300, 1024])
@pytest.mark.parametrize("name", sorted(MANY_CASES))
def test_attend_many_requests(form, parts, name):
    check(*attend(form, MANY_CASES[name], parts=parts, D=256 if form == "latent" else 64))


@pytest.mark.parametrize("form", ["latent", "expanded"])
@pytest.mark.parametrize("parts", [0, 3, 50])
@pytest.mark.parametrize("what", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("name", sorted(POISON_CASES))
def test_attend_values_that_a_row_does_not_see(form, parts, what, name):
    """A value that is not finite reaches the rows that see its key, and no others.  In the latent form the value is
    part of the key, whose score is then not finite either: rows that see it are NaN (or, where the score is -inf,
    as without it but for 0 * inf), and only the others are compared."""
    c = POISON_CASES[name]
    x = float(what)
    kv, nq = c["kv"][0], c["nq"][0]
    keys = [kv - 1, kv - 3, max(0, kv - nq - 2), max(0, kv - nq - 25)]

    def poison_pool(rows, rows64, table):
        for t in keys:
            rows[table[0, t // 16], t % 16, 5 + t % 7] = x

    def poison_rows(ex, ex64, kv_base):
        for t in keys:
            ex[kv_base[0] + t, :, ex.shape[2] // 2 + 5 + t % 7] = x

    got = attend(form, c, parts=parts, poison=poison_pool if form == "latent" else poison_rows)
    seen = ref.seen_keys(kv, nq, True, c.get("window", 0), np.ones(kv, dtype=bool))[:, keys].any(1)
    rows = np.ones(got[0].shape[0], dtype=bool)
    rows[:nq][seen] = False
    check(*[a[rows] for a in got[:5]], got[5])
    if form == "expanded":
        for i in np.flatnonzero(seen):
            per = ref.seen_keys(kv, nq, True, c.get("window", 0), np.ones(kv, dtype=bool))[i]
            cols = sorted({5 + t % 7 for t in keys if per[t]})
            want = np.zeros(got[0].shape[2], dtype=bool)
            want[cols] = True
            for h in range(c["H"]):
                np.testing.assert_array_equal(~np.isfinite(got[0][i, h]), want)
                if what != "nan":
                    assert (got[0][i, h, cols] == x).all()


def weightless(form, kv, nq, keys, parts, alone=False):
    """One request of `nq` queries of 4 heads over `kv` keys, of which `keys` (with `alone` all) have a weight of 0 and
    a value in column 5 that is not finite: got out, got lse, and what the other keys give (as `attend` does), seen."""
    rng = np.random.default_rng(11)
    H, D = 4, 256 if form == "latent" else 64
    table, pool = table_for(rng, [kv], 16)
    rows, rows64 = bf16(rng.standard_normal((pool, 16, (D if form == "latent" else 256) + 64)))
    q, _ = bf16(rng.standard_normal((nq, H, D + 64)))
    ex, ex64 = bf16(rng.standard_normal((kv, H, 2 * D)))
    keys = list(range(kv)) if alone else keys
    if form == "latent":                           # the score is -infinity by the value itself
        q[..., 5] = 1.0
        for t in keys:
            rows[table[0, t // 16], t % 16, 5] = -float("inf")
    else:                                          # far below the others', or -infinity
        q[..., 0] = 8.0
        ex[..., 0], ex64[..., 0] = 0.0, 0.0
        for t in keys:
            ex[t, :, 0], ex[t, :, D + 5] = -float("inf") if alone else -30000.0, float("inf")
    q64 = values(q)
    out, lse = torch.zeros(nq, H, D, dtype=torch.bfloat16, device=DEV), torch.zeros(nq, H, device=DEV)
    kw = dict(n_queries=nq, n_keys=kv, scale=0.08, lse=lse, n_parts=parts)
    if form == "latent":
        km.attend_latent(q, rows, out, i32(table), i32([kv]), **kw)
    else:
        km.attend_expanded(q, ex[..., :D], ex[..., D:], rows[..., -64:], out, i32(table), i32([kv]), **kw)
    x, ok = ref.gather(rows64, table[0], kv, 16)
    seen = ref.seen_keys(kv, nq, True, 0, ok)
    rest = seen.copy()
    rest[:, keys] = False
    if form == "latent":
        k, v = x[None], x[None, :, :D]
    else:
        e = ex64.transpose(1, 0, 2)
        k, v = np.concatenate([e[..., :D], np.broadcast_to(x[None, :, -64:], (H, kv, 64))], -1), e[..., D:]
    want, size, want_lse, most = ref.attend_rows(q64, k, v, rest, 0.08)
    return values(out), values(lse), want, size, want_lse, most * (D + 64 + 8) * 2.0 ** -24, seen[:, keys].any(1)


@pytest.mark.parametrize("form", ["latent", "expanded"])
@pytest.mark.parametrize("parts", [0, 1, 3, 50])
@pytest.mark.parametrize("keys", [[10], [291], [40, 100, 285]])
@pytest.mark.parametrize("nq", [2, 20])
def test_attend_a_value_that_is_not_finite_with_no_weight(form, parts, keys, nq):
    """A key that a row sees with a weight of 0, in steps that all rows see whole and in others: its value that is not
    finite leaves that column not finite, whatever divides the keys, and nothing else of the row."""
    *got, seen = weightless(form, 300, nq, keys, parts)
    assert not np.isfinite(got[0][seen][..., 5]).any()
    assert np.isfinite(got[0][~seen]).all()
    got[0][seen, :, 5], got[2][seen, :, 5] = 0.0, 0.0
    check(*got)


@pytest.mark.parametrize("form", ["latent", "expanded"])
@pytest.mark.parametrize("parts", [0, 1, 9])
@pytest.mark.parametrize("kv,nq", [(1, 1), (5, 3), (70, 1), (200, 40)])
def test_attend_rows_whose_every_score_is_minus_infinity(form, parts, kv, nq):
    """They get 0 and an lse of -infinity, but for a column whose values are not finite."""
    out, lse = weightless(form, kv, nq, [], parts, alone=True)[:2]
    assert not np.isfinite(out[..., 5]).any()
    assert (out[..., :5] == 0).all() and (out[..., 6:] == 0).all()
    assert (lse == -np.inf).all()


@pytest.mark.parametrize("parts", [0, 3, 50])
@pytest.mark.parametrize("name", sorted(POISON_CASES))
@pytest.mark.parametrize("what", ["nan", "inf", "-inf"])
def test_attend_latent_values_arrive_at_the_rows_that_see_them(name, what, parts):
    """A NaN in a pool row makes its score NaN, and so the whole of every row that sees it; an infinity makes its column
    not finite there."""
    c = POISON_CASES[name]
    kv, nq = c["kv"][0], c["nq"][0]
    keys = [kv - 1, kv - 3, max(0, kv - nq - 2), max(0, kv - nq - 25)]

    def poison(rows, rows64, table):
        for t in keys:
            rows[table[0, t // 16], t % 16, 5 + t % 7] = float(what)

    got, lse = attend("latent", c, parts=parts, poison=poison)[:2]
    per = ref.seen_keys(kv, nq, True, c.get("window", 0), np.ones(kv, dtype=bool))[:, keys]
    assert per.any()
    for i in np.flatnonzero(per.any(1)):
        if what == "nan":
            assert np.isnan(got[i]).all() and np.isnan(lse[i]).all()
        else:
            assert not np.isfinite(got[i][:, sorted({5 + t % 7 for t, there in zip(keys, per[i]) if there})]).any()


@pytest.mark.parametrize("form", ["latent", "expanded"])
def test_attend_a_query_that_is_not_finite_stays_in_its_row(form):
    torch.manual_seed(0)
    pool = torch.randn(8, 16, 576, device=DEV).to(torch.bfloat16)
    table, kv = i32([[1, 5, 2, 7, 0]]), i32([75])
    D = 512 if form == "latent" else 128
    q = torch.randn(20, 16, D + 64, device=DEV).to(torch.bfloat16)
    ex = torch.randn(75, 16, 256, device=DEV).to(torch.bfloat16)

    def call(q):
        out = torch.zeros(20, 16, D, dtype=torch.bfloat16, device=DEV)
        kw = dict(n_queries=20, n_keys=75, scale=0.05)
        if form == "latent":
            km.attend_latent(q, pool, out, table, kv, **kw)
        else:
            km.attend_expanded(q, ex[..., :128], ex[..., 128:], pool[..., 512:], out, table, kv, **kw)
        return out

    want = call(q)
    bad = q.clone()
    bad[3, 7, 100], bad[11, 0, D + 5] = float("nan"), float("inf")
    got = call(bad)
    assert got[3, 7].isnan().all() and got[11, 0].isnan().all()
    got[3, 7], got[11, 0] = want[3, 7], want[11, 0]
    assert torch.equal(got, want)


def test_attend_views():
    """Tensors in other orders and inside wider ones give the same bits as packed ones: heads outermost, tokens of
    all layers side by side, pages in reverse of the allocation, results and sums between other columns."""
    rng = np.random.default_rng(4)
    kv, nq, H = [300, 90], [5, 20], 6
    table, pages = table_for(rng, kv, 16)
    table, base, n = i32(table), i32([0, 5]), 25
    rand = lambda *shape: bf16(rng.standard_normal(shape))[0]
    wide = rand(16, pages, 3, 640)                 # token, page, layer, columns
    cache = wide[:, :, 1, 32:608].transpose(0, 1)
    q = rand(H, n, 648)[..., 8:584].transpose(0, 1)
    ex = rand(H, sum(kv), 264)[..., 8:].transpose(0, 1)
    kw = dict(n_queries=20, n_keys=300, scale=0.05, q_base=base, q_tokens=i32(nq))
    for parts in (0, 9):
        kw["n_parts"] = parts
        out = [torch.full((H, n, 528), 7.0, dtype=torch.bfloat16, device=DEV), torch.zeros(n, H, 512, dtype=torch.bfloat16, device=DEV)]
        lse = [torch.full((H, 2, n), 7.0, device=DEV), torch.zeros(n, H, device=DEV)]
        km.attend_latent(q, cache, out[0][..., 8:520].transpose(0, 1), table, i32(kv), lse=lse[0][:, 1].transpose(0, 1), **kw)
        km.attend_latent(q.contiguous(), cache.contiguous(), out[1], table, i32(kv), lse=lse[1], **kw)
        assert torch.equal(out[0][..., 8:520].transpose(0, 1), out[1]) and out[1].abs().sum() > 0
        assert torch.equal(lse[0][:, 1].transpose(0, 1), lse[1])
        assert (out[0][..., :8] == 7.0).all() and (out[0][..., 520:] == 7.0).all() and (lse[0][:, 0] == 7.0).all()
        out = [torch.full((H, n, 144), 7.0, dtype=torch.bfloat16, device=DEV), torch.zeros(n, H, 128, dtype=torch.bfloat16, device=DEV)]
        kx = dict(kw, kv_base=i32([0, 300]))
        km.attend_expanded(q[..., :192], ex[..., 128:], ex[..., :128], cache[..., 512:], out[0][..., 8:136].transpose(0, 1), table,
                           i32(kv), lse=lse[0][:, 1].transpose(0, 1), **kx)
        km.attend_expanded(q[..., :192].contiguous(), ex[..., 128:].contiguous(), ex[..., :128].contiguous(),
                           cache[..., 512:].contiguous(), out[1], table, i32(kv), lse=lse[1], **kx)
        assert torch.equal(out[0][..., 8:136].transpose(0, 1), out[1]) and out[1].abs().sum() > 0
        assert torch.equal(lse[0][:, 1].transpose(0, 1), lse[1])
        assert (out[0][..., :8] == 7.0).all() and (out[0][..., 136:] == 7.0).all()
    # one key and value for all heads (a head stride of 0), as heads of their own
    one = [torch.zeros(n, H, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    k1 = ex[:, :1, 128:].expand(-1, H, -1)
    km.attend_expanded(q[..., :192], k1, k1, cache[..., 512:], one[0], table, i32(kv), **kx)
    km.attend_expanded(q[..., :192], k1.contiguous(), k1.contiguous(), cache[..., 512:], one[1], table, i32(kv), **kx)
    assert torch.equal(*one) and one[0].abs().sum() > 0


def test_expand_views():
    """The pool's columns from a wider row, W shared by all heads, results with heads outermost."""
    rng = np.random.default_rng(6)
    kv, H = [200, 1, 70], 3
    table, pages = table_for(rng, kv, 16)
    rand = lambda *shape: bf16(rng.standard_normal(shape))[0]
    cache = rand(16, pages, 2, 640)[:, :, 1, 64:].transpose(0, 1)
    for w in (rand(H, 512, 192), rand(1, 512, 256).expand(H, -1, -1), rand(H, 192, 512).transpose(1, 2)):
        out = [torch.full((H, 271, w.shape[2] + 16), 7.0, dtype=torch.bfloat16, device=DEV),
               torch.zeros(271, H, w.shape[2], dtype=torch.bfloat16, device=DEV)]
        kw = dict(n_keys=200, row_base=i32([0, 200, 201]))
        view = out[0][..., 8:-8].transpose(0, 1)
        km.expand_latent(cache, w, view, i32(table), i32(kv), **kw)
        km.expand_latent(cache.contiguous(), w.contiguous(), out[1], i32(table), i32(kv), **kw)
        # the two orders of W sum the same products in the same order
        assert torch.equal(view, out[1]) and out[1].abs().sum() > 0
        assert (out[0][..., :8] == 7.0).all() and (out[0][..., -8:] == 7.0).all()


@pytest.mark.parametrize("form", ["latent", "expanded"])
def test_attend_repeats_bit_for_bit(form):
    for name in ("long", "chunk"):
        a = attend(form, ATTEND_CASES[name])
        b = attend(form, ATTEND_CASES[name])
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


@pytest.mark.parametrize("form", ["latent", "expanded"])
def test_parts_of_a_context_join_by_lse(form):
    """Attention over the first and the last pages of a context, joined by lse, is attention over all of it."""
    torch.manual_seed(3)
    pool = torch.randn(20, 16, 576, device=DEV).to(torch.bfloat16)
    D = 512 if form == "latent" else 128
    q = torch.randn(2, 16, D + 64, device=DEV).to(torch.bfloat16)
    ex = torch.randn(320, 16, 256, device=DEV).to(torch.bfloat16)
    table = torch.arange(20, dtype=torch.int32, device=DEV)[None]

    def call(first, n):
        out, lse = torch.zeros(2, 16, D, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 16, device=DEV)
        kw = dict(n_queries=2, n_keys=n, scale=0.05, causal=False, lse=lse)
        t = table[:, first // 16:]
        if form == "latent":
            km.attend_latent(q, pool, out, t, i32([n]), **kw)
        else:
            km.attend_expanded(q, ex[first:, :, :128], ex[first:, :, 128:], pool[..., 512:], out, t, i32([n]),
                               kv_base=i32([0]), **kw)
        return out.double(), lse.double()

    (a, la), (b, lb), (w, lw) = call(0, 112), call(112, 208), call(0, 320)
    both = torch.logaddexp(la, lb)
    got = a * (la - both).exp()[..., None] + b * (lb - both).exp()[..., None]
    assert (got - w).abs().max() <= 2 * 4 * U * w.abs().max()
    assert (both - lw).abs().max() < 1e-4


def test_cache_offsets_past_32_bits():
    """Pool pages, expanded rows and outputs past 2^32 bytes."""
    torch.manual_seed(4)
    pages = (1 << 32) // (16 * 1152) + 40
    pool = torch.zeros(pages, 16, 576, dtype=torch.bfloat16, device=DEV)
    table = i32([[pages - 1, 3, pages - 7], [pages - 20, pages - 2, 5]])
    kv = i32([47, 33])
    idx = table.long()
    pool[idx] = torch.randn(2, 3, 16, 576, device=DEV).to(torch.bfloat16)
    small = torch.zeros(6, 16, 576, dtype=torch.bfloat16, device=DEV)
    small[:] = pool[idx].view(6, 16, 576)
    near = i32([[0, 1, 2], [3, 4, 5]])
    q = torch.randn(4, 16, 576, device=DEV).to(torch.bfloat16)
    outs = []
    for p, t in ((pool, table), (small, near)):
        out = torch.zeros(4, 16, 512, dtype=torch.bfloat16, device=DEV)
        km.attend_latent(q, p, out, t, kv, n_queries=2, n_keys=47, scale=0.05)
        outs.append(out)
    assert torch.equal(*outs)
    w = torch.randn(2, 512, 256, device=DEV).to(torch.bfloat16)
    far = torch.zeros((1 << 32) // 1024 + 100, 2, 256, dtype=torch.bfloat16, device=DEV)
    at = far.shape[0] - 90
    km.expand_latent(pool, w, far, table, kv, n_keys=47, row_base=i32([at, 0]))
    out = torch.zeros(94, 2, 256, dtype=torch.bfloat16, device=DEV)
    km.expand_latent(small, w, out, near, kv, n_keys=47)
    assert torch.equal(far[at:at + 47], out[:47]) and torch.equal(far[:33], out[47:80])
    q2 = torch.randn(4, 2, 192, device=DEV).to(torch.bfloat16)
    got = [torch.zeros(4, 2, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    km.attend_expanded(q2, far[..., :128], far[..., 128:], pool[..., 512:], got[0], table, kv, n_queries=2, n_keys=47,
                       scale=0.05, kv_base=i32([at, 0]))
    km.attend_expanded(q2, out[..., :128], out[..., 128:], small[..., 512:], got[1], near, kv, n_queries=2, n_keys=47,
                       scale=0.05)
    assert torch.equal(*got)
    rows = torch.randn(1, 2, 20, 1, 576, device=DEV).to(torch.bfloat16).transpose(0, 1)
    km.append_rotated(rows, None, pool[None, :, :, None], None, table, rope=km.RopeSpec(theta=1e4, rope_dim=64, rope_offset=512),
                      tokens_before=i32([10, 12]))
    km.append_rotated(rows, None, small[None, :, :, None], None, near, rope=km.RopeSpec(theta=1e4, rope_dim=64, rope_offset=512),
                      tokens_before=i32([10, 12]))
    assert torch.equal(pool[idx].view(6, 16, 576), small)


# ---------------------------------------------------------------------------
# together, as they are used
# ---------------------------------------------------------------------------

class Layer:
    """One latent-attention layer: rows from seeded projections, both forms of attention."""

    def __init__(self, heads=16, pages=40, page=16, seed=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.H, self.page, self.gen = heads, page, g
        self.rope = km.RopeSpec(theta=1e4, rope_dim=64, rope_offset=512, pairing="interleaved")
        self.pool = torch.full((pages, page, 576), float("nan"), dtype=torch.bfloat16, device=DEV)
        # one weight as a checkpoint has it: [heads, keys and values, latent]
        self.w = self.rand(heads, 256, 512, std=512 ** -0.5)
        self.scale = 192 ** -0.5

    def rand(self, *shape, std=1.0):
        return (torch.randn(shape, generator=self.gen, device=DEV) * std).to(torch.bfloat16)

    def append(self, rows, q, q_lat, table, before, n, base):
        km.append_rotated(rows[None, :, None], None, self.pool[None, :, :, None], None, table, rope=self.rope,
                          n_tokens=n, tokens_before=before, row_base=base, q=q[None, :, :, 128:], q_out=q_lat[None, :, :, 512:])

    def absorbed(self, q, q_lat, table, kv, n, n_keys, o_lat, out, **kw):
        km.project_heads(q[..., :128], self.w[:, :128], q_lat[..., :512])
        km.attend_latent(q_lat, self.pool, o_lat, table, kv, n_queries=n, n_keys=n_keys, scale=self.scale, **kw)
        km.project_heads(o_lat, self.w[:, 128:].transpose(1, 2), out)

    def expanded(self, q, q_lat, table, kv, n, n_keys, out, **kw):
        rows = torch.empty(kv.shape[0] * n_keys, self.H, 256, dtype=torch.bfloat16, device=DEV)
        km.expand_latent(self.pool, self.w.transpose(1, 2), rows, table, kv, n_keys=n_keys)
        q = torch.cat([q[..., :128], q_lat[..., 512:]], -1)
        km.attend_expanded(q, rows[..., :128], rows[..., 128:], self.pool[..., 512:], out, table, kv, n_queries=n,
                           n_keys=n_keys, scale=self.scale, **kw)


def test_absorbed_and_expanded_forms_agree():
    """A prompt of two requests through both forms.  The absorbed form rounds q Wk and the latent result to bf16, the
    expanded one keys and values: scores differ by a few u of sum |q k| scale / sqrt(128), outputs by a few u."""
    y = Layer()
    n, table, kv = 75, i32([[3, 9, 1, 17, 5], [20, 8, 30, 2, 11]]), i32([75, 75])
    q, q_lat = y.rand(150, 16, 192), torch.zeros(150, 16, 576, dtype=torch.bfloat16, device=DEV)
    y.append(y.rand(150, 576), q, q_lat, table, i32([0, 0]), n, i32([0, 75]))
    o_lat = torch.zeros(150, 16, 512, dtype=torch.bfloat16, device=DEV)
    a, b = (torch.zeros(150, 16, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    y.absorbed(q, q_lat, table, kv, n, 75, o_lat, a)
    y.expanded(q, q_lat, table, kv, n, 75, b)
    # against 64 bits from the rows in the pool
    x = y.pool[table.long()].view(2, 80, 576)[:, :75].double().cpu()
    w, qq = y.w.double().cpu(), torch.cat([q[..., :128], q_lat[..., 512:]], -1).double().cpu().view(2, 75, 16, 192)
    k = torch.cat([torch.matmul(x[:, None, :, :512], w[:, :128].transpose(1, 2)), x[:, None, :, 512:].expand(-1, 16, -1, -1)], -1)
    v = torch.matmul(x[:, None, :, :512], w[:, 128:].transpose(1, 2))
    s = torch.matmul(qq.transpose(1, 2), k.transpose(2, 3)) * y.scale
    s = s.masked_fill(torch.ones(75, 75, dtype=torch.bool).triu(1), float("-inf"))
    p = torch.softmax(s, -1)
    want = torch.matmul(p, v).transpose(1, 2).reshape(150, 16, 128)
    size = torch.matmul(p, v.abs()).transpose(1, 2).reshape(150, 16, 128)
    # |score| errors: u sum |q||k| scale, at most u * 192 * max |q k| * scale; observed spread of s bounds it here
    e = float(2 * U * (torch.matmul(qq.abs().transpose(1, 2), k.abs().transpose(2, 3)) * y.scale).max())
    for got in (a, b):
        err = (got.double().cpu() - want).abs()
        assert (err <= (4 * U + 2 * e) * size).all(), float((err / size).max())


def decode(y, steps, graph, stream=None):
    """Tokens one by one through the absorbed form, captured or not; outputs of every step."""
    R, H = 3, y.H
    table = torch.arange(R * 10, dtype=torch.int32, device=DEV).view(R, 10)
    before, kv = i32([20, 0, 31]), i32([21, 1, 32])
    y.pool[:] = y.rand(*y.pool.shape)
    rows, q = torch.zeros(R, 576, dtype=torch.bfloat16, device=DEV), torch.zeros(R, H, 192, dtype=torch.bfloat16, device=DEV)
    q_lat, o_lat = (torch.zeros(R, H, d, dtype=torch.bfloat16, device=DEV) for d in (576, 512))
    out, base = torch.zeros(R, H, 128, dtype=torch.bfloat16, device=DEV), i32([0, 1, 2])
    lse = torch.zeros(R, H, device=DEV)

    def step():
        y.append(rows, q, q_lat, table, before, 1, base)
        y.absorbed(q, q_lat, table, kv, 1, 160, o_lat, out, lse=lse, n_parts=5)
        before.add_(1)
        kv.add_(1)

    g = None
    if graph:
        step()                                     # warm, then back
        before.sub_(1), kv.sub_(1)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
    got = []
    for _ in range(steps):
        rows.copy_(y.rand(*rows.shape)), q.copy_(y.rand(*q.shape))
        g.replay() if g is not None else step()
        got.append(out.clone())
        if len(got) % 3 == 0:
            torch.cuda.synchronize()
            torch.matmul(torch.ones(64, 64, device=DEV), torch.ones(64, 64, device=DEV))
    torch.cuda.synchronize()
    return torch.stack(got)


def test_decode_loop_and_captured_replays():
    eager, captured = decode(Layer(seed=5), 9, False), decode(Layer(seed=5), 9, True)
    assert torch.isfinite(eager.float()).all()
    assert torch.equal(eager, captured)


def test_two_captured_graphs_with_workspaces_of_their_own():
    """Each prepared call has a workspace of its own: replays in turn do not meet."""
    torch.manual_seed(9)
    pool = torch.randn(64, 16, 576, device=DEV).to(torch.bfloat16)
    table, kv = torch.arange(64, dtype=torch.int32, device=DEV)[None], i32([1000])
    qs = [torch.randn(1, 16, 576, device=DEV).to(torch.bfloat16) for _ in range(2)]
    outs = [torch.zeros(1, 16, 512, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    calls = [km.prepare_attend_latent(q, pool, o, table, kv, n_queries=1, n_keys=1024, scale=0.05) for q, o in zip(qs, outs)]
    assert calls[0].workspace is not None and calls[0].workspace.data_ptr() != calls[1].workspace.data_ptr()
    for c in calls:
        c.launch()
    want = [o.clone() for o in outs]
    graphs = []
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.launch()
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(4):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_calls_on_a_given_stream():
    """Every call runs on the stream that it is given, behind that stream's work."""
    torch.manual_seed(2)
    pool = torch.randn(64, 16, 576, device=DEV).to(torch.bfloat16)
    table, kv = torch.arange(64, dtype=torch.int32, device=DEV)[None], i32([1000])
    q = torch.randn(1, 16, 576, device=DEV).to(torch.bfloat16)
    w = torch.randn(16, 512, 256, device=DEV).to(torch.bfloat16)
    o = {s: torch.zeros(1, 16, 512, dtype=torch.bfloat16, device=DEV) for s in "ab"}
    e = {s: torch.zeros(1024, 16, 256, dtype=torch.bfloat16, device=DEV) for s in "ab"}
    r = {s: torch.zeros(1, 16, 256, dtype=torch.bfloat16, device=DEV) for s in "ab"}
    x = {s: torch.zeros(1, 16, 128, dtype=torch.bfloat16, device=DEV) for s in "ab"}
    torch.cuda.synchronize()
    s1 = torch.cuda.Stream()
    for name, st in (("a", None), ("b", s1)):
        km.attend_latent(q, pool, o[name], table, kv, n_queries=1, n_keys=1024, scale=0.05, stream=st)
        km.expand_latent(pool, w, e[name], table, kv, n_keys=1024, stream=st)
        km.project_heads(o[name], w, r[name], stream=st)
        km.attend_expanded(q[..., :192], e[name][..., :128], e[name][..., 128:], pool[..., 512:], x[name], table, kv,
                           n_queries=1, n_keys=1024, scale=0.05, stream=st)
    torch.cuda.synchronize()
    for d in (o, e, r, x):
        assert torch.equal(d["a"], d["b"]) and d["a"].abs().sum() > 0


@pytest.mark.parametrize("heads", [16, 40])
def test_prompt_and_decode_over_recalled_rows(heads):
    """Two chunks rebuilt by rehydrate at their new places, a question behind them and a token behind that: rows in the
    pool, both forms of attention and the products, each link in 64 bits from what it was handed."""
    y = Layer(heads=heads, seed=3)
    n, nq, H = 48, 20, heads
    chunks = y.rand(2, 1, n, 1, 576)
    table = i32([[7, 2, 31, 4, 0, 9, 12, 30]])     # the chunks' pages, then the question's
    km.rehydrate(chunks, y.pool.view(1, -1, 1, 576), rope=y.rope, chunk_pos=i32([[0] * 3, [n] * 3]),
                 page_table=table[0, :6].view(2, 3).contiguous(), page_size=16, n_pool_pages=y.pool.shape[0])
    new, q = y.rand(nq + 1, 576), y.rand(nq + 1, H, 192)
    q_lat = torch.zeros(nq + 1, H, 576, dtype=torch.bfloat16, device=DEV)
    o_lat = torch.zeros(nq + 1, H, 512, dtype=torch.bfloat16, device=DEV)
    out = torch.zeros(nq + 1, H, 128, dtype=torch.bfloat16, device=DEV)
    rows = torch.zeros(128, H, 256, dtype=torch.bfloat16, device=DEV)
    a, b = slice(0, nq), slice(nq, nq + 1)         # the question, in the expanded form; the token, in the absorbed one
    y.append(new[a], q[a], q_lat[a], table, i32([2 * n]), nq, i32([0]))
    km.expand_latent(y.pool, y.w.transpose(1, 2), rows, table, i32([2 * n + nq]), n_keys=128)
    q_exp = torch.cat([q[a, :, :128], q_lat[a, :, 512:]], -1)
    lse = torch.zeros(nq + 1, H, device=DEV)
    km.attend_expanded(q_exp, rows[..., :128], rows[..., 128:], y.pool[..., 512:], out[a], table, i32([2 * n + nq]),
                       n_queries=nq, n_keys=128, scale=y.scale, lse=lse[a])
    y.append(new[b], q[b], q_lat[b], table, i32([2 * n + nq]), 1, i32([0]))
    y.absorbed(q[b], q_lat[b], table, i32([2 * n + nq + 1]), 1, 128, o_lat[b], out[b], lse=lse[b])
    torch.cuda.synchronize()

    kv = 2 * n + nq + 1
    pool = values(y.pool[table[0].long()]).reshape(128, 576)
    src = np.concatenate([values(chunks).reshape(2 * n, 576), values(new)])
    f = ref.frequencies(1e4, 64)
    for t in range(kv):
        r, size = ref.rotate(src[t, 512:], t * f, "interleaved")
        assert (np.abs(pool[t, 512:] - r) <= U * np.abs(r) + 2.0 ** -18 * size).all()
    np.testing.assert_array_equal(pool[:kv, :512], src[:, :512])
    for i in range(nq + 1):
        r, size = ref.rotate(values(q[i, :, 128:]), (2 * n + i) * f, "interleaved")
        assert (np.abs(values(q_lat[i, :, 512:]) - r) <= U * np.abs(r) + 2.0 ** -18 * size).all()
    w, ex = values(y.w), values(rows)
    for h in range(H):
        for got, x, m in ((ex[:kv - 1, h], pool[:kv - 1, :512], w[h].T), (values(q_lat[b, h, :512]), values(q[b, h, :128]), w[h, :128]),
                          (values(out[b, h]), values(o_lat[b, h]), w[h, 128:].T)):
            want, tol = product_bound(x, m)
            assert (np.abs(got - want) <= tol).all()
    e = ex[:kv - 1].transpose(1, 0, 2)
    k = np.concatenate([e[..., :128], np.broadcast_to(pool[None, :kv - 1, 512:], (H, kv - 1, 64))], -1)
    seen = ref.seen_keys(kv - 1, nq, True, 0, np.ones(kv - 1, dtype=bool))
    want = ref.attend_rows(values(q_exp), k, e[..., 128:], seen, y.scale)
    check(values(out[a]), values(lse[a]), *want[:3], want[3] * (192 + 8) * 2.0 ** -24)
    want = ref.attend_rows(values(q_lat[b]), pool[None, :kv], pool[None, :kv, :512], np.ones((1, kv), dtype=bool), y.scale)
    check(values(o_lat[b]), values(lse[b]), *want[:3], want[3] * (576 + 8) * 2.0 ** -24)
