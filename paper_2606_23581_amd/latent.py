"""Serving from a paged latent cache: rows of a latent and a rope key, one for all
heads of a token, as ``rehydrate`` puts them into the pool.

Binding of the entry points of the same names in ``include/kamera.h``; the
package re-exports everything here.  As elsewhere in the package each call has a
``prepare_`` form that returns a ``Prepared`` call for a program whose buffers
stay in place.

* ``append_rotated``   new rows into the bf16 paged pool, rotary positions applied
                       on the way, with the rope bands of their queries
* ``project_heads``    a product with a matrix of its own for every head: queries
                       into the latent's columns, results out of them
* ``expand_latent``    every head's keys and values from the pool's latents
* ``attend_latent``    attention over the pool's rows themselves (absorbed form)
* ``attend_expanded``  attention over expanded keys and values
"""

from __future__ import annotations

import ctypes
import dataclasses

from . import CRope, Prepared, RopeSpec, _bf16, _check, _i32, _i64, _ptr, _vp, lib
from .cache import _device, _inner, _int, _launch_on, _table, _typed, _workspace

SCALING_NONE = 0
SCALING_LINEAR = 1
SCALING_TURNS = 2
SCALING_PAIRS = 3

_f64 = ctypes.c_double
_f32 = ctypes.c_float


class CRopeScaling(ctypes.Structure):
    _fields_ = [("kind", _i32), ("factor", _f64), ("original_tokens", _f64), ("low_turns", _f64),
                ("high_turns", _f64), ("amplitude", _f64)]


class CAppendRotatedArgs(ctypes.Structure):
    _fields_ = [("n_chunks", _i32), ("n_layers", _i32), ("n_tokens", _i32), ("n_k_heads", _i32), ("k_dim", _i32),
                ("n_v_heads", _i32), ("v_dim", _i32), ("n_q_heads", _i32), ("page_size", _i32), ("pt_stride", _i32),
                ("pt_pages", _i32), ("n_pool_pages", _i32), ("rope", CRope), ("scaling", CRopeScaling),
                ("chunk_tokens", _vp), ("tokens_before", _vp), ("row_base", _vp), ("page_table", _vp),
                ("positions", _vp), ("position_stride", _i64 * 3), ("k", _vp), ("k_stride", _i64 * 4), ("v", _vp),
                ("v_stride", _i64 * 4), ("q", _vp), ("q_stride", _i64 * 4), ("q_out", _vp), ("q_out_stride", _i64 * 4),
                ("k_cache", _vp), ("k_cache_stride", _i64 * 4), ("v_cache", _vp), ("v_cache_stride", _i64 * 4),
                ("status", _vp)]


class CProjectArgs(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("n_heads", _i32), ("n_in", _i32), ("n_out", _i32), ("x", _vp), ("x_stride", _i64 * 2),
                ("w", _vp), ("w_stride", _i64 * 3), ("out", _vp), ("out_stride", _i64 * 2)]


class CExpandArgs(ctypes.Structure):
    _fields_ = [("n_requests", _i32), ("n_heads", _i32), ("n_in", _i32), ("n_out", _i32), ("n_keys", _i32),
                ("page_size", _i32), ("pt_stride", _i32), ("n_pool_pages", _i32), ("kv_tokens", _vp),
                ("row_base", _vp), ("page_table", _vp), ("cache", _vp), ("cache_stride", _i64 * 2), ("w", _vp),
                ("w_stride", _i64 * 3), ("out", _vp), ("out_stride", _i64 * 2), ("status", _vp)]


class CAttendLatentArgs(ctypes.Structure):
    _fields_ = [("n_requests", _i32), ("n_heads", _i32), ("latent_dim", _i32), ("rope_dim", _i32), ("n_queries", _i32),
                ("n_keys", _i32), ("page_size", _i32), ("pt_stride", _i32), ("n_pool_pages", _i32), ("causal", _i32),
                ("window", _i32), ("scale", _f32), ("n_parts", _i32), ("q_tokens", _vp), ("q_base", _vp),
                ("kv_tokens", _vp), ("page_table", _vp), ("q", _vp), ("q_stride", _i64 * 2), ("out", _vp),
                ("out_stride", _i64 * 2), ("lse", _vp), ("lse_stride", _i64 * 2), ("cache", _vp),
                ("cache_stride", _i64 * 2), ("workspace", _vp), ("workspace_bytes", _i64), ("status", _vp)]


class CAttendExpandedArgs(ctypes.Structure):
    _fields_ = [("n_requests", _i32), ("n_heads", _i32), ("head_dim", _i32), ("rope_dim", _i32), ("n_queries", _i32),
                ("n_keys", _i32), ("page_size", _i32), ("pt_stride", _i32), ("n_pool_pages", _i32), ("causal", _i32),
                ("window", _i32), ("scale", _f32), ("n_parts", _i32), ("q_tokens", _vp), ("q_base", _vp),
                ("kv_tokens", _vp), ("kv_base", _vp), ("page_table", _vp), ("q", _vp), ("q_stride", _i64 * 2),
                ("out", _vp), ("out_stride", _i64 * 2), ("lse", _vp), ("lse_stride", _i64 * 2), ("k", _vp),
                ("k_stride", _i64 * 2), ("v", _vp), ("v_stride", _i64 * 2), ("rope_cache", _vp),
                ("rope_cache_stride", _i64 * 2), ("workspace", _vp), ("workspace_bytes", _i64), ("status", _vp)]


STRUCTS = {10: CAppendRotatedArgs, 11: CProjectArgs, 12: CExpandArgs, 13: CAttendLatentArgs, 14: CAttendExpandedArgs}
EXPORTS = ("kamera_append_rotated", "kamera_project_heads", "kamera_expand_latent", "kamera_attend_latent",
           "kamera_attend_expanded", "kamera_attend_latent_workspace", "kamera_attend_expanded_workspace",
           "kamera_validate_latent")


def declare(L) -> None:
    """Signatures of this module's entry points on the loaded library."""
    for name, cls in (("kamera_append_rotated", CAppendRotatedArgs), ("kamera_project_heads", CProjectArgs),
                      ("kamera_expand_latent", CExpandArgs), ("kamera_attend_latent", CAttendLatentArgs),
                      ("kamera_attend_expanded", CAttendExpandedArgs)):
        fn = getattr(L, name)
        fn.argtypes = [ctypes.POINTER(cls), _vp]
        fn.restype = _i32
    for name, cls in (("kamera_attend_latent_workspace", CAttendLatentArgs),
                      ("kamera_attend_expanded_workspace", CAttendExpandedArgs)):
        fn = getattr(L, name)
        fn.argtypes = [ctypes.POINTER(cls)]
        fn.restype = _i64
    L.kamera_validate_latent.argtypes = [_i32, _vp]
    L.kamera_validate_latent.restype = _i32


@dataclasses.dataclass(frozen=True)
class RopeScaling:
    """Rotary positions scaled for contexts longer than ``original_tokens`` by ``factor``: "linear" for all pairs,
    "turns" or "pairs" only for those that turn rarely over the original context (fewer than ``low_turns`` times:
    fully; more than ``high_turns``: not at all; between by turns or by the pair's number).  Rotated columns are
    multiplied by ``amplitude``."""

    kind: str
    factor: float
    original_tokens: float = 0.0
    low_turns: float = 1.0
    high_turns: float = 32.0
    amplitude: float = 1.0

    def to_c(self) -> CRopeScaling:
        kinds = {"linear": SCALING_LINEAR, "turns": SCALING_TURNS, "pairs": SCALING_PAIRS}
        if self.amplitude == 0.0:
            raise ValueError("amplitude must not be 0")
        return CRopeScaling(kinds[self.kind], float(self.factor), float(self.original_tokens), float(self.low_turns),
                            float(self.high_turns), float(self.amplitude))


def append_rotated(*a, stream=None, **kw) -> None:
    """``kamera_append_rotated``; see ``prepare_append_rotated`` for the arguments."""
    prepare_append_rotated(*a, **kw).launch(stream)


def prepare_append_rotated(k, v, k_cache, v_cache, page_table, *, rope: RopeSpec, scaling: RopeScaling = None,
                           positions=None, n_tokens: int = None, tokens_before=None, chunk_tokens=None,
                           row_base=None, q=None, q_out=None, status=None) -> Prepared:
    """bf16 rows into the bf16 paged pool behind the tokens that each chunk has there, keys rotated at their
    positions, and the rope bands of their queries.

    k: [C, L, n, H, D] (any strides, last dim contiguous), or with row_base (int32 [C]) [L, rows, H, D], chunk
    c's rows from row_base[c] on and at most n_tokens of them.  k_cache: [L, pages, page_size, H, D].  v, v_cache:
    the same with heads and columns of their own, or None (latent rows).  page_table: int32 [C, pages of a chunk],
    also columns of a wider table: a chunk ends (STATUS_BAD_LENGTH) where its row of the view does.
    q, q_out: views of the queries' bands alone, [C, L, n, heads, rope_dim] or [L, rows, heads, rope_dim]; q_out
    may be q.  positions: int32 [C, n, coordinates] or [rows, coordinates] (3 with sections, else 1, or without
    that dimension); default the tokens' places in the cache.  tokens_before, chunk_tokens: int32 [C] (default 0
    and all rows).
    """
    import torch

    L = lib()
    C = page_table.shape[0]
    packed = row_base is not None
    coords = 1 if rope.sections is None else 3
    if packed and n_tokens is None:
        raise ValueError("with row_base, n_tokens is given")
    a = CAppendRotatedArgs()
    a.rope = rope.to_c()
    if scaling is not None:
        a.scaling = scaling.to_c()

    def rows(t, name, field):
        _inner(_bf16(t, name), name)
        if t.dim() != (4 if packed else 5) or (not packed and t.shape[0] != C):
            raise ValueError(f"{name} must be " + ("[L, rows, H, D]" if packed else f"[{C}, L, n, H, D]"))
        field[0:4] = (0, *t.stride()[:3]) if packed else t.stride()[:4]
        return t.shape[-4:]

    Ln, n_rows, H, D = rows(k, "k", a.k_stride)
    n = n_rows if n_tokens is None else _int(n_tokens, "n_tokens")
    if n > n_rows:
        raise ValueError(f"n_tokens {n} exceeds the {n_rows} rows of k")

    def pool(t, name, field, heads, dim):
        _inner(_bf16(t, name), name)
        if t.dim() != 5 or t.shape[0] != Ln or tuple(t.shape[3:]) != (heads, dim):
            raise ValueError(f"{name} must be [{Ln}, pages, page_size, {heads}, {dim}] (got {tuple(t.shape)})")
        field[0:4] = t.stride()[:4]
        return t.shape[1:3]

    n_pages, page_size = pool(k_cache, "k_cache", a.k_cache_stride, H, D)
    if (v is None) != (v_cache is None):
        raise ValueError("v and v_cache go together")
    if v is not None:
        vl, vn, a.n_v_heads, a.v_dim = rows(v, "v", a.v_stride)
        if (vl, vn) != (Ln, n_rows):
            raise ValueError("k and v must have the same layers and rows")
        if pool(v_cache, "v_cache", a.v_cache_stride, a.n_v_heads, a.v_dim) != (n_pages, page_size):
            raise ValueError("k_cache and v_cache must have the same pages")
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    if q is not None:
        ql, qn, a.n_q_heads, qd = rows(q, "q", a.q_stride)
        rows(q_out, "q_out", a.q_out_stride)
        if q_out.shape != q.shape or (ql, qn) != (Ln, n_rows) or qd != rope.rope_dim:
            raise ValueError(f"q and q_out must be the bands of k's rows, {rope.rope_dim} columns")
    if positions is not None:
        _typed(positions, torch.int32, "positions", contiguous=False)
        lead = (n_rows,) if packed else (C, n_rows)
        if tuple(positions.shape) != (*lead, coords) and not (coords == 1 and tuple(positions.shape) == lead):
            raise ValueError(f"positions must be {list((*lead, coords))} (got {tuple(positions.shape)})")
        st = positions.stride()
        st = st if len(st) > len(lead) else (*st, 0)
        a.position_stride[0:3] = (0, *st) if packed else st
    for t, nm in ((tokens_before, "tokens_before"), (chunk_tokens, "chunk_tokens"), (row_base, "row_base")):
        _typed(t, torch.int32, nm, (C,))
    _typed(status, torch.int32, "status")
    a.n_chunks, a.n_layers, a.n_tokens, a.n_k_heads, a.k_dim = C, Ln, n, H, D
    # chunks may outgrow the rows of a view: they end where the view does
    a.page_size, a.pt_stride, a.pt_pages, a.n_pool_pages = page_size, _table(page_table, C, 0), page_table.shape[1], n_pages
    _device(k, v, q, q_out, k_cache, v_cache, page_table, positions, tokens_before, chunk_tokens, row_base, status)
    a.chunk_tokens, a.tokens_before, a.row_base = _ptr(chunk_tokens), _ptr(tokens_before), _ptr(row_base)
    a.page_table, a.positions = _ptr(page_table), _ptr(positions)
    a.k, a.v, a.q, a.q_out = _ptr(k), _ptr(v), _ptr(q), _ptr(q_out)
    a.k_cache, a.v_cache, a.status = _ptr(k_cache), _ptr(v_cache), _ptr(status)
    return Prepared(L.kamera_append_rotated, a, (k, v, k_cache, v_cache, page_table, positions, tokens_before,
                                                 chunk_tokens, row_base, q, q_out, status))


def _weights(a, w, heads):
    """w [heads, in, out], one of the last two dimensions contiguous, entered into the arguments."""
    _bf16(w, "w")
    if w.dim() != 3 or w.shape[0] != heads:
        raise ValueError(f"w must be [{heads}, in, out] (got {tuple(w.shape)})")
    a.n_in, a.n_out = w.shape[1:]
    a.w = _ptr(w)
    a.w_stride[0:3] = w.stride()


def project_heads(*a, stream=None, **kw) -> None:
    """``kamera_project_heads``; see ``prepare_project_heads`` for the arguments."""
    prepare_project_heads(*a, **kw).launch(stream)


def prepare_project_heads(x, w, out) -> Prepared:
    """out[i, g] = x[i, g] @ w[g].

    x: bf16 [rows, H, in] (also expanded over the heads); w: bf16 [H, in, out], the inputs or the outputs
    contiguous (a transposed view); out: bf16 [rows, H, out].
    """
    L = lib()
    _inner(_bf16(x, "x"), "x"), _inner(_bf16(out, "out"), "out")
    if x.dim() != 3:
        raise ValueError(f"x must be [rows, heads, in] (got {tuple(x.shape)})")
    a = CProjectArgs()
    n, H, width = x.shape
    _weights(a, w, H)
    if a.n_in != width or tuple(out.shape) != (n, H, a.n_out):
        raise ValueError(f"x [{n}, {H}, {width}], w {tuple(w.shape)} and out {tuple(out.shape)} do not fit")
    _device(x, w, out)
    a.n_rows, a.n_heads, a.x, a.out = _int(n, "rows"), H, _ptr(x), _ptr(out)
    a.x_stride[0:2], a.out_stride[0:2] = x.stride()[:2], out.stride()[:2]
    return Prepared(L.kamera_project_heads, a, (x, w, out))


def _pool_rows(cache, name, width=None):
    """A pool's rows as [pages, page_size, columns]."""
    _inner(_bf16(cache, name), name)
    if cache.dim() != 3 or (width is not None and cache.shape[2] != width):
        raise ValueError(f"{name} must be [pages, page_size, {'columns' if width is None else width}] (got {tuple(cache.shape)})")
    return cache.shape


def expand_latent(*a, stream=None, **kw) -> None:
    """``kamera_expand_latent``; see ``prepare_expand_latent`` for the arguments."""
    prepare_expand_latent(*a, **kw).launch(stream)


def prepare_expand_latent(cache, w, out, page_table, kv_tokens, *, n_keys: int, row_base=None, status=None) -> Prepared:
    """out[row_base[r] + t, g] = (the first w.shape[1] columns of token t's pool row) @ w[g].

    cache: bf16 [pages, page_size, columns], one layer of the pool; w: bf16 [H, in, out] as in
    ``prepare_project_heads``; out: bf16 [rows, H, out]; page_table: int32 [R, pages]; kv_tokens: int32 [R], at
    most n_keys; row_base: int32 [R] (default r * n_keys).
    """
    import torch

    L = lib()
    n_pages, page_size, columns = _pool_rows(cache, "cache")
    _inner(_bf16(out, "out"), "out")
    R = kv_tokens.shape[0]
    a = CExpandArgs()
    if out.dim() != 3:
        raise ValueError(f"out must be [rows, heads, out] (got {tuple(out.shape)})")
    _weights(a, w, out.shape[1])
    if a.n_in > columns or out.shape[2] != a.n_out:
        raise ValueError(f"cache {tuple(cache.shape)}, w {tuple(w.shape)} and out {tuple(out.shape)} do not fit")
    a.n_keys = _int(n_keys, "n_keys")
    if row_base is None and R * a.n_keys > out.shape[0]:
        raise ValueError(f"{R} requests of {a.n_keys} tokens exceed the {out.shape[0]} rows of out")
    _typed(kv_tokens, torch.int32, "kv_tokens", (R,)), _typed(row_base, torch.int32, "row_base", (R,))
    _typed(status, torch.int32, "status")
    a.n_requests, a.n_heads, a.page_size, a.n_pool_pages = R, out.shape[1], page_size, n_pages
    a.pt_stride = _table(page_table, R, a.n_keys, page_size)
    _device(cache, w, out, page_table, kv_tokens, row_base, status)
    a.kv_tokens, a.row_base, a.page_table = _ptr(kv_tokens), _ptr(row_base), _ptr(page_table)
    a.cache, a.out, a.status = _ptr(cache), _ptr(out), _ptr(status)
    a.cache_stride[0:2], a.out_stride[0:2] = cache.stride()[:2], out.stride()[:2]
    return Prepared(L.kamera_expand_latent, a, (cache, w, out, page_table, kv_tokens, row_base, status))


def _attend_args(a, q, out, page_table, kv_tokens, page_size, n_pages, n_queries, n_keys, scale, causal, window, n_parts,
                 q_base, q_tokens, lse, status):
    """What both forms of attention take alike."""
    import torch

    R, rows = kv_tokens.shape[0], q.shape[0]
    a.n_requests, a.n_heads, a.n_queries, a.n_keys = R, q.shape[1], _int(n_queries, "n_queries"), _int(n_keys, "n_keys")
    if q_base is None and R * a.n_queries > rows:
        raise ValueError(f"{R} requests of {a.n_queries} queries exceed the {rows} rows of q")
    for t, nm in ((kv_tokens, "kv_tokens"), (q_base, "q_base"), (q_tokens, "q_tokens")):
        _typed(t, torch.int32, nm, (R,))
    _typed(lse, torch.float32, "lse", (rows, q.shape[1]), contiguous=False)
    _typed(status, torch.int32, "status")
    a.page_size, a.n_pool_pages, a.pt_stride = page_size, n_pages, _table(page_table, R, a.n_keys, page_size)
    # a window past 32 bits holds every key there can be
    a.causal, a.window, a.n_parts = int(causal), _int(min(window, (1 << 31) - 1), "window"), _int(n_parts, "n_parts")
    a.scale = float(scale)
    a.q_tokens, a.q_base, a.kv_tokens, a.page_table = _ptr(q_tokens), _ptr(q_base), _ptr(kv_tokens), _ptr(page_table)
    a.q, a.out, a.lse, a.status = _ptr(q), _ptr(out), _ptr(lse), _ptr(status)
    a.q_stride[0:2], a.out_stride[0:2] = q.stride()[:2], out.stride()[:2]
    if lse is not None:
        a.lse_stride[0:2] = lse.stride()


def attend_latent(*a, stream=None, **kw) -> None:
    """``kamera_attend_latent``; see ``prepare_attend_latent`` for the arguments."""
    _launch_on(stream, prepare_attend_latent, a, kw)


def prepare_attend_latent(q, cache, out, page_table, kv_tokens, *, n_queries: int, n_keys: int, scale: float,
                          q_base=None, q_tokens=None, causal: bool = True, window: int = 0, lse=None, workspace=None,
                          n_parts: int = 0, status=None) -> Prepared:
    """Attention of a batch of requests over the rows of one layer of a paged latent pool.

    q: bf16 [rows, heads, latent + 64], queries in the latent's columns with their rotated bands behind;
    cache: bf16 [pages, page_size, latent + 64]; out: bf16 [rows, heads, latent].  Request r's query tokens are
    rows q_base[r] + i (r * n_queries + i without q_base), q_tokens[r] of them (default n_queries).
    page_table: int32 [R, pages]; kv_tokens: int32 [R], tokens in the pool, at most n_keys.  scale: of the scores.
    window > 0: only the last `window` keys up to a query's own.  lse: fp32 [rows, heads], receives the log of
    the softmax sums.  workspace: as in ``prepare_attend_paged``.
    """
    L = lib()
    _inner(_bf16(q, "q"), "q"), _inner(_bf16(out, "out"), "out")
    if q.dim() != 3 or out.dim() != 3 or out.shape[:2] != q.shape[:2]:
        raise ValueError("q and out must be [rows, heads, columns] with the same rows and heads")
    n_pages, page_size, _ = _pool_rows(cache, "cache", q.shape[2])
    a = CAttendLatentArgs()
    a.latent_dim, a.rope_dim = out.shape[2], q.shape[2] - out.shape[2]
    _attend_args(a, q, out, page_table, kv_tokens, page_size, n_pages, n_queries, n_keys, scale, causal, window, n_parts,
                 q_base, q_tokens, lse, status)
    a.cache = _ptr(cache)
    a.cache_stride[0:2] = cache.stride()[:2]
    workspace = _workspace(a, L.kamera_attend_latent_workspace(ctypes.byref(a)), workspace, q.device)
    _device(q, cache, out, page_table, kv_tokens, q_base, q_tokens, lse, workspace, status)
    call = Prepared(L.kamera_attend_latent, a, (q, cache, out, page_table, kv_tokens, q_base, q_tokens, lse, workspace,
                                                status))
    call.workspace = workspace
    return call


def attend_expanded(*a, stream=None, **kw) -> None:
    """``kamera_attend_expanded``; see ``prepare_attend_expanded`` for the arguments."""
    _launch_on(stream, prepare_attend_expanded, a, kw)


def prepare_attend_expanded(q, k, v, rope_cache, out, page_table, kv_tokens, *, n_queries: int, n_keys: int,
                            scale: float, kv_base=None, q_base=None, q_tokens=None, causal: bool = True,
                            window: int = 0, lse=None, workspace=None, n_parts: int = 0, status=None) -> Prepared:
    """Attention over expanded keys and values, the rope keys read from the pool.

    q: bf16 [rows, heads, D + 64]; k, v: bf16 [kv rows, heads, D] as ``expand_latent`` writes them (views of one
    tensor), request r's from row kv_base[r] on (int32 [R], default r * n_keys); rope_cache: bf16 [pages,
    page_size, 64], the pool's last columns; out: bf16 [rows, heads, D].  Everything else as in
    ``prepare_attend_latent``.
    """
    import torch

    L = lib()
    for t, nm in ((q, "q"), (k, "k"), (v, "v"), (out, "out")):
        _inner(_bf16(t, nm), nm)
        if t.dim() != 3:
            raise ValueError(f"{nm} must be [rows, heads, columns] (got {tuple(t.shape)})")
    if out.shape[:2] != q.shape[:2] or k.shape != v.shape or tuple(k.shape[1:]) != tuple(out.shape[1:]):
        raise ValueError("q and out must have the same rows and heads, k, v and out the same heads and columns")
    a = CAttendExpandedArgs()
    a.head_dim, a.rope_dim = out.shape[2], q.shape[2] - out.shape[2]
    n_pages, page_size, _ = _pool_rows(rope_cache, "rope_cache", a.rope_dim)
    R = kv_tokens.shape[0]
    _typed(kv_base, torch.int32, "kv_base", (R,))
    _attend_args(a, q, out, page_table, kv_tokens, page_size, n_pages, n_queries, n_keys, scale, causal, window, n_parts,
                 q_base, q_tokens, lse, status)
    if kv_base is None and R * a.n_keys > k.shape[0]:
        raise ValueError(f"{R} requests of {a.n_keys} keys exceed the {k.shape[0]} rows of k")
    a.kv_base, a.k, a.v, a.rope_cache = _ptr(kv_base), _ptr(k), _ptr(v), _ptr(rope_cache)
    a.k_stride[0:2], a.v_stride[0:2] = k.stride()[:2], v.stride()[:2]
    a.rope_cache_stride[0:2] = rope_cache.stride()[:2]
    workspace = _workspace(a, L.kamera_attend_expanded_workspace(ctypes.byref(a)), workspace, q.device)
    _device(q, k, v, rope_cache, out, page_table, kv_tokens, kv_base, q_base, q_tokens, lse, workspace, status)
    call = Prepared(L.kamera_attend_expanded, a, (q, k, v, rope_cache, out, page_table, kv_tokens, kv_base, q_base,
                                                  q_tokens, lse, workspace, status))
    call.workspace = workspace
    return call


__all__ = ["SCALING_NONE", "SCALING_LINEAR", "SCALING_TURNS", "SCALING_PAIRS", "CRopeScaling", "CAppendRotatedArgs",
           "CProjectArgs", "CExpandArgs", "CAttendLatentArgs", "CAttendExpandedArgs", "RopeScaling", "append_rotated",
           "prepare_append_rotated", "project_heads", "prepare_project_heads", "expand_latent",
           "prepare_expand_latent", "attend_latent", "prepare_attend_latent", "attend_expanded",
           "prepare_attend_expanded"]
