"""Serving from the paged cache: pages for requests, the cache in 8 bits, and
attention over it.

Binding of the entry points of the same names in ``include/kamera.h``; the
package re-exports everything here.  As elsewhere in the package each call has a
``prepare_`` form that returns a ``Prepared`` call for a program whose buffers
stay in place.

* ``page_tables``    pages from a free list and token slots for growing requests
* ``append_paged8``  bf16 K, V rows into the 8-bit cache (e4m3, a power-of-two
                     scale for each page and head), with the pages' key sums
* ``select_pages``   the pages a query needs most, by an integer score
* ``attend_paged``   attention over the paged cache, 8 bits or bf16
"""

from __future__ import annotations

import ctypes
import dataclasses

from . import Prepared, _bf16, _check, _i32, _i32_dev, _i64, _ptr, _stream, _vp, lib

STATUS_NO_PAGE = 2
STATUS_BAD_LENGTH = 4
MAX_REQUESTS = 8192
MAX_SELECT_PAGES = 32768
MAX_GROUP = 64
CACHE_BF16 = 0
CACHE_E4M3 = 1


class CPageTablesArgs(ctypes.Structure):
    _fields_ = [("n_requests", _i32), ("page_size", _i32), ("pt_stride", _i32), ("n_pool_pages", _i32),
                ("tokens_before", _vp), ("tokens_after", _vp), ("free_pages", _vp), ("n_free", _i32),
                ("free_begin", _vp), ("free_end", _vp), ("page_table", _vp), ("token_base", _vp), ("slots", _vp),
                ("n_slots", _i64), ("status", _vp)]


class CAppendArgs(ctypes.Structure):
    _fields_ = [("n_chunks", _i32), ("n_layers", _i32), ("n_heads", _i32), ("head_dim", _i32), ("n_tokens", _i32),
                ("page_size", _i32), ("pt_stride", _i32), ("n_pool_pages", _i32), ("chunk_tokens", _vp),
                ("tokens_before", _vp), ("row_base", _vp), ("page_table", _vp), ("k", _vp), ("k_stride", _i64 * 4),
                ("v", _vp), ("v_stride", _i64 * 4), ("k_cache", _vp), ("k_cache_stride", _i64 * 4), ("v_cache", _vp),
                ("v_cache_stride", _i64 * 4), ("k_scale", _vp), ("k_scale_stride", _i64 * 3), ("v_scale", _vp),
                ("v_scale_stride", _i64 * 3), ("k_sum", _vp), ("k_sum_stride", _i64 * 3), ("k_sum_scale", _vp),
                ("k_sum_scale_stride", _i64 * 3), ("status", _vp), ("pt_pages", _i32)]


class CSelectArgs(ctypes.Structure):
    _fields_ = [("n_requests", _i32), ("n_q_heads", _i32), ("n_kv_heads", _i32), ("head_dim", _i32), ("n_keys", _i32),
                ("page_size", _i32), ("pt_stride", _i32), ("n_pool_pages", _i32), ("kv_tokens", _vp),
                ("page_table", _vp), ("q", _vp), ("q_stride", _i64 * 2), ("k_sum", _vp), ("k_sum_stride", _i64 * 2),
                ("k_sum_scale", _vp), ("k_sum_scale_stride", _i64 * 2), ("n_keep", _i32), ("n_first", _i32),
                ("n_last", _i32), ("sel", _vp), ("sel_count", _vp), ("workspace", _vp), ("workspace_bytes", _i64),
                ("status", _vp)]


class CAttendArgs(ctypes.Structure):
    _fields_ = [("n_requests", _i32), ("n_q_heads", _i32), ("n_kv_heads", _i32), ("head_dim", _i32),
                ("n_queries", _i32), ("n_keys", _i32), ("page_size", _i32), ("pt_stride", _i32),
                ("n_pool_pages", _i32), ("cache_type", _i32), ("causal", _i32), ("window", _i32),
                ("scale", ctypes.c_float), ("n_splits", _i32), ("q_tokens", _vp), ("q_base", _vp), ("kv_tokens", _vp),
                ("page_table", _vp), ("q", _vp), ("q_stride", _i64 * 2), ("out", _vp), ("out_stride", _i64 * 2),
                ("lse", _vp), ("lse_stride", _i64 * 2), ("k_cache", _vp), ("k_cache_stride", _i64 * 3),
                ("v_cache", _vp), ("v_cache_stride", _i64 * 3), ("k_scale", _vp), ("k_scale_stride", _i64 * 2),
                ("v_scale", _vp), ("v_scale_stride", _i64 * 2), ("sel", _vp), ("sel_count", _vp), ("sel_stride", _i32),
                ("pt_pages", _i32), ("workspace", _vp), ("workspace_bytes", _i64), ("status", _vp)]


STRUCTS = {6: CPageTablesArgs, 7: CAppendArgs, 8: CSelectArgs, 9: CAttendArgs}
EXPORTS = ("kamera_page_tables", "kamera_append_paged8", "kamera_select_pages", "kamera_attend_paged",
           "kamera_attend_workspace", "kamera_select_workspace", "kamera_validate_cache")


def declare(L) -> None:
    """Signatures of this module's entry points on the loaded library."""
    for name, cls in (("kamera_page_tables", CPageTablesArgs), ("kamera_append_paged8", CAppendArgs),
                      ("kamera_select_pages", CSelectArgs), ("kamera_attend_paged", CAttendArgs)):
        fn = getattr(L, name)
        fn.argtypes = [ctypes.POINTER(cls), _vp]
        fn.restype = _i32
    L.kamera_attend_workspace.argtypes = [ctypes.POINTER(CAttendArgs)]
    L.kamera_attend_workspace.restype = _i64
    L.kamera_select_workspace.argtypes = [ctypes.POINTER(CSelectArgs)]
    L.kamera_select_workspace.restype = _i64
    L.kamera_validate_cache.argtypes = [_i32, _vp]
    L.kamera_validate_cache.restype = _i32


def _typed(t, dtype, name, shape=None, contiguous=True):
    """t (or None) checked for its type, shape and, by default, dense layout."""
    if t is None:
        return None
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {str(dtype).replace('torch.', '')} (got {t.dtype})")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _int(x, name) -> int:
    """x as the library takes it, in 32 bits (the binding's structs would keep its low ones)."""
    x = int(x)
    if not -(1 << 31) <= x < 1 << 31:
        raise ValueError(f"{name} must fit in 32 bits (got {x})")
    return x


def _table(page_table, n, tokens=None, page_size=1):
    """The row stride of an int32 [n, pages] table whose rows are dense.

    Where that is more than the rows of this view hold, a call says how many tokens a request has at most, and none
    of the rest is looked up (0 where the library is told the pages of a row itself); a call that cannot say
    (tokens None) needs the rest of the last row to be there too.
    """
    _i32_dev(page_table, "page_table")
    shape = page_table.shape
    if len(shape) != 2 or shape[0] != n:
        raise ValueError(f"page_table must be [{n}, pages] (got {tuple(shape)})")
    s0, s1 = page_table.stride()
    if s1 != 1 and shape[1] > 1 and n > 0:
        raise ValueError("the rows of page_table must be contiguous")
    if n <= 1:
        return max(shape[1], 1)
    if s0 > shape[1]:
        if tokens is not None and tokens > shape[1] * page_size:
            raise ValueError(f"the {shape[1]} pages of a row of page_table hold less than {tokens} tokens")
        there = page_table.untyped_storage().nbytes() // 4 - page_table.storage_offset()
        if tokens is None and n * s0 > there:
            raise ValueError("the rows of page_table must be whole")
    return s0


def _device(*tensors):
    """All tensors on one GPU."""
    dev = None
    for t in tensors:
        if t is not None and t.device != dev:
            if dev is not None:
                raise ValueError(f"tensors on {dev} and {t.device} in one call")
            dev = t.device
            if dev.type != "cuda":
                raise ValueError("tensors must be in device memory")


def _workspace(a, need, workspace, device):
    """The given workspace, or one of `need` bytes (or none), entered into the arguments."""
    import torch

    _check(min(need, 0))
    if need > 0 and workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    if workspace is not None:
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        a.workspace, a.workspace_bytes = _ptr(workspace), workspace.numel() * workspace.element_size()
    return workspace


def _launch_on(stream, prepare, a, kw) -> None:
    """Prepares and launches a call that may have a workspace of its own: memory of the stream that it runs on,
    which other work of the current stream may still use otherwise."""
    if stream is None:
        prepare(*a, **kw).launch()
        return
    import torch

    s, handle = stream, _stream(stream)
    if not isinstance(s, torch.cuda.Stream):         # a raw handle, or an object that has one
        s = torch.cuda.ExternalStream(handle) if handle else torch.cuda.default_stream()
    with torch.cuda.stream(s):
        prepare(*a, **kw).launch(s)


def _is8(t):
    import torch

    return t.dtype is torch.float8_e4m3fn or t.dtype is torch.uint8


def _inner(t, name):
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"the innermost dimension of {name} must be contiguous")
    return t


# ---------------------------------------------------------------------------

@dataclasses.dataclass
class Cache8:
    """An 8-bit paged cache of n_layers layers: K and V as views [layers, pages, page_size, heads, dim] of
    memory that keeps what one (page, head) needs together, their scales [layers, pages, heads], and the
    pages' key sums.  ``layer(l)`` is one layer's part as the keyword arguments that ``attend_paged`` takes."""

    k: "object"
    v: "object"
    k_scale: "object"
    v_scale: "object"
    k_sum: "object"
    k_sum_scale: "object"

    @staticmethod
    def allocate(n_layers: int, n_pages: int, page_size: int, n_heads: int, head_dim: int, device="cuda") -> "Cache8":
        import torch

        def plane():
            x = torch.zeros((n_layers, n_pages, n_heads, page_size, head_dim), dtype=torch.uint8, device=device)
            return x.view(torch.float8_e4m3fn).transpose(2, 3)

        def per_head():
            return torch.ones((n_layers, n_pages, n_heads), dtype=torch.float32, device=device)

        return Cache8(plane(), plane(), per_head(), per_head(),
                      torch.zeros((n_layers, n_pages, n_heads, head_dim), dtype=torch.int8, device=device), per_head())

    def layer(self, l: int) -> dict:
        return {"k_cache": self.k[l], "v_cache": self.v[l], "k_scale": self.k_scale[l], "v_scale": self.v_scale[l]}


def page_tables(*a, stream=None, **kw) -> None:
    """``kamera_page_tables``; see ``prepare_page_tables`` for the arguments."""
    prepare_page_tables(*a, **kw).launch(stream)


def prepare_page_tables(tokens_before, tokens_after, free_pages, page_table, *, page_size: int, n_pool_pages: int,
                        free_end, token_base, free_begin=None, slots=None, status=None) -> Prepared:
    """Pages and slots for requests that grow from tokens_before (or None: 0) to tokens_after tokens.

    tokens_*: int32 [R]; free_pages: int32 [F], taken in order from free_begin[0] (0 if None) on;
    page_table: int32 [R, pages], new pages are entered; free_end: int32 [1], receives the first place
    of the list not taken; token_base: int32 [R + 1], receives the sums of new tokens; slots: int64 [n],
    receives the slot of every new token, -1 after them.
    """
    import torch

    L = lib()
    R = tokens_after.shape[0]
    a = CPageTablesArgs()
    a.n_requests, a.page_size = R, _int(page_size, "page_size")
    a.n_pool_pages = _int(n_pool_pages, "n_pool_pages")
    i32 = torch.int32
    _typed(tokens_before, i32, "tokens_before", (R,)), _typed(tokens_after, i32, "tokens_after", (R,))
    _typed(free_pages, i32, "free_pages"), _typed(free_begin, i32, "free_begin", (1,))
    _typed(free_end, i32, "free_end", (1,)), _typed(token_base, i32, "token_base", (R + 1,))
    _typed(status, i32, "status")
    _typed(slots, torch.int64, "slots")
    _device(tokens_before, tokens_after, free_pages, page_table, free_begin, free_end, token_base, slots, status)
    a.pt_stride = _table(page_table, R)
    if R > 1 and a.pt_stride != page_table.shape[1]:
        raise ValueError("page_table must be contiguous")
    a.tokens_before, a.tokens_after = _ptr(tokens_before), _ptr(tokens_after)
    a.free_pages, a.n_free = _ptr(free_pages), int(free_pages.numel())
    a.free_begin, a.free_end = _ptr(free_begin), _ptr(free_end)
    a.page_table, a.token_base = _ptr(page_table), _ptr(token_base)
    if slots is not None:
        a.slots, a.n_slots = _ptr(slots), int(slots.numel())
    a.status = _ptr(status)
    return Prepared(L.kamera_page_tables, a, (tokens_before, tokens_after, free_pages, page_table, free_begin,
                                              free_end, token_base, slots, status))


def append_paged8(*a, stream=None, **kw) -> None:
    """``kamera_append_paged8``; see ``prepare_append_paged8`` for the arguments."""
    prepare_append_paged8(*a, **kw).launch(stream)


def prepare_append_paged8(k, v, k_cache, v_cache, k_scale, v_scale, page_table, *, n_tokens: int = None,
                          tokens_before=None, chunk_tokens=None, row_base=None, k_sum=None, k_sum_scale=None,
                          status=None) -> Prepared:
    """bf16 rows into the 8-bit paged cache, behind the tokens that each chunk has there.

    k, v: [C, L, n, H, D] (any strides, last dim contiguous), or with row_base (int32 [C]) [L, rows, H, D],
    chunk c's rows from row_base[c] on and at most n_tokens of them.  k_cache, v_cache: float8_e4m3fn (or
    uint8) [L, pages, page_size, H, D]; k_scale, v_scale: fp32 [L, pages, H]; k_sum: int8 [L, pages, H, D]
    with k_sum_scale fp32 [L, pages, H] (optional).  page_table: int32 [C, pages of a chunk], also columns of a
    wider table: a chunk ends (STATUS_BAD_LENGTH) where its row of the view does.
    tokens_before, chunk_tokens: int32 [C] (default 0 and all rows).
    """
    import torch

    L = lib()
    _inner(_bf16(k, "k"), "k"), _inner(_bf16(v, "v"), "v")
    a = CAppendArgs()
    if k.shape != v.shape:
        raise ValueError("k and v must have one shape")
    C = page_table.shape[0]
    if row_base is not None:
        if k.dim() != 4 or n_tokens is None:
            raise ValueError("with row_base, k and v are [L, rows, H, D] and n_tokens is given")
        Ln, _, H, D = k.shape
        a.k_stride[0:4] = (0, *k.stride()[:3])
        a.v_stride[0:4] = (0, *v.stride()[:3])
        n = _int(n_tokens, "n_tokens")
    else:
        if k.dim() != 5 or k.shape[0] != C:
            raise ValueError("k and v must be [C, L, n, H, D], C the rows of page_table")
        _, Ln, rows, H, D = k.shape
        a.k_stride[0:4] = k.stride()[:4]
        a.v_stride[0:4] = v.stride()[:4]
        n = rows if n_tokens is None else _int(n_tokens, "n_tokens")
        if n > rows:
            raise ValueError(f"n_tokens {n} exceeds the {rows} rows of a chunk")
    if k_cache.dim() != 5 or k_cache.shape != v_cache.shape:
        raise ValueError("k_cache and v_cache must be [L, pages, page_size, H, D]")
    _, n_pages, page_size = k_cache.shape[:3]
    if k_cache.shape != (Ln, n_pages, page_size, H, D):
        raise ValueError(f"the caches must be [{Ln}, pages, page_size, {H}, {D}] (got {tuple(k_cache.shape)})")
    for t, nm in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        if not _is8(t):
            raise TypeError(f"{nm} must be float8_e4m3fn or uint8 (got {t.dtype})")
        _inner(t, nm)
    for t, nm in ((k_scale, "k_scale"), (v_scale, "v_scale"), (k_sum_scale, "k_sum_scale")):
        _typed(t, torch.float32, nm, (Ln, n_pages, H), contiguous=False)
    _typed(k_sum, torch.int8, "k_sum", (Ln, n_pages, H, D), contiguous=False)
    for t, nm in ((tokens_before, "tokens_before"), (chunk_tokens, "chunk_tokens"), (row_base, "row_base")):
        _typed(t, torch.int32, nm, (C,))
    _typed(status, torch.int32, "status")
    _device(k, v, k_cache, v_cache, k_scale, v_scale, page_table, tokens_before, chunk_tokens, row_base, k_sum,
            k_sum_scale, status)
    a.n_chunks, a.n_layers, a.n_heads, a.head_dim, a.n_tokens = C, Ln, H, D, n
    # chunks may outgrow the rows of a view: they end where the view does
    a.page_size, a.pt_stride, a.n_pool_pages = page_size, _table(page_table, C, 0), n_pages
    a.pt_pages = page_table.shape[1]
    a.chunk_tokens, a.tokens_before, a.row_base = _ptr(chunk_tokens), _ptr(tokens_before), _ptr(row_base)
    a.page_table, a.k, a.v = _ptr(page_table), _ptr(k), _ptr(v)
    a.k_cache, a.v_cache, a.k_scale, a.v_scale = _ptr(k_cache), _ptr(v_cache), _ptr(k_scale), _ptr(v_scale)
    a.k_cache_stride[0:4] = k_cache.stride()[:4]
    a.v_cache_stride[0:4] = v_cache.stride()[:4]
    a.k_scale_stride[:] = k_scale.stride()
    a.v_scale_stride[:] = v_scale.stride()
    if k_sum is not None:
        _inner(k_sum, "k_sum")
        a.k_sum = _ptr(k_sum)
        a.k_sum_stride[0:3] = k_sum.stride()[:3]
    if k_sum_scale is not None:
        a.k_sum_scale = _ptr(k_sum_scale)
        a.k_sum_scale_stride[:] = k_sum_scale.stride()
    a.status = _ptr(status)
    return Prepared(L.kamera_append_paged8, a, (k, v, k_cache, v_cache, k_scale, v_scale, page_table, tokens_before,
                                                chunk_tokens, row_base, k_sum, k_sum_scale, status))


def select_pages(*a, stream=None, **kw) -> None:
    """``kamera_select_pages``; see ``prepare_select_pages`` for the arguments."""
    _launch_on(stream, prepare_select_pages, a, kw)


def prepare_select_pages(q, k_sum, k_sum_scale, page_table, kv_tokens, sel, sel_count, *, n_keys: int,
                         page_size: int, n_first: int = 1, n_last: int = 1, workspace=None,
                         status=None) -> Prepared:
    """The sel.shape[-1] pages of each request that its query needs most, for every KV head.

    q: bf16 [R, heads, D], one query token a request; k_sum: int8 [pages, H, D] and k_sum_scale: fp32
    [pages, H], one layer's key sums; page_table: int32 [R, pages]; kv_tokens: int32 [R], at most n_keys.
    sel: int32 [R, H, keep], receives ascending page indices (-1 after them), sel_count: int32 [R, H].
    The first n_first and the last n_last pages are always taken.  workspace: as in ``prepare_attend_paged``.
    """
    import torch

    L = lib()
    _inner(_bf16(q, "q"), "q")
    R, HQ, D = q.shape
    _inner(_typed(k_sum, torch.int8, "k_sum", contiguous=False), "k_sum")
    n_pages, H = k_sum.shape[:2]
    if k_sum.shape[2] != D:
        raise ValueError("q and k_sum must have one head size")
    _typed(k_sum_scale, torch.float32, "k_sum_scale", (n_pages, H), contiguous=False)
    _typed(kv_tokens, torch.int32, "kv_tokens", (R,))
    keep = sel.shape[-1]
    _typed(sel, torch.int32, "sel", (R, H, keep))
    _typed(sel_count, torch.int32, "sel_count", (R, H))
    _typed(status, torch.int32, "status")
    _device(q, k_sum, k_sum_scale, page_table, kv_tokens, sel, sel_count, workspace, status)
    a = CSelectArgs()
    a.n_requests, a.n_q_heads, a.n_kv_heads, a.head_dim, a.n_keys = R, HQ, H, D, _int(n_keys, "n_keys")
    a.page_size, a.n_pool_pages = _int(page_size, "page_size"), n_pages
    a.pt_stride = _table(page_table, R, a.n_keys, a.page_size)
    a.kv_tokens, a.page_table, a.q = _ptr(kv_tokens), _ptr(page_table), _ptr(q)
    a.q_stride[0:2] = q.stride()[:2]
    a.k_sum, a.k_sum_scale = _ptr(k_sum), _ptr(k_sum_scale)
    a.k_sum_stride[0:2] = k_sum.stride()[:2]
    a.k_sum_scale_stride[:] = k_sum_scale.stride()
    a.n_keep, a.n_first, a.n_last = keep, _int(n_first, "n_first"), _int(n_last, "n_last")
    a.sel, a.sel_count, a.status = _ptr(sel), _ptr(sel_count), _ptr(status)
    workspace = _workspace(a, L.kamera_select_workspace(ctypes.byref(a)), workspace, q.device)
    call = Prepared(L.kamera_select_pages, a, (q, k_sum, k_sum_scale, page_table, kv_tokens, sel, sel_count,
                                               workspace, status))
    call.workspace = workspace
    return call


def attend_paged(*a, stream=None, **kw) -> None:
    """``kamera_attend_paged``; see ``prepare_attend_paged`` for the arguments."""
    _launch_on(stream, prepare_attend_paged, a, kw)


def attend_workspace(prepared: Prepared) -> int:
    """``kamera_attend_workspace`` of a prepared attention call: bytes, 0 where the work is not split."""
    n = lib().kamera_attend_workspace(ctypes.byref(prepared.args))
    _check(min(n, 0))
    return n


def prepare_attend_paged(q, k_cache, v_cache, out, page_table, kv_tokens, *, n_queries: int, n_keys: int,
                         q_base=None, q_tokens=None, k_scale=None, v_scale=None, scale: float = None,
                         causal: bool = True, window: int = 0, sel=None, sel_count=None, lse=None, workspace=None,
                         n_splits: int = 0, status=None) -> Prepared:
    """Attention of a batch of requests over one layer of the paged cache.

    q, out: bf16 [rows, heads, D]; request r's query tokens are rows q_base[r] + i (r * n_queries + i
    without q_base), q_tokens[r] of them (default n_queries).  k_cache, v_cache: one layer, [pages,
    page_size, H, D], bf16, or float8_e4m3fn / uint8 with k_scale, v_scale fp32 [pages, H].
    page_table: int32 [R, pages]; kv_tokens: int32 [R], tokens in the cache, at most n_keys.
    scale: of the scores, default D ** -0.5.  window > 0: only the last `window` keys up to a query's own.
    sel, sel_count: int32 [R, H, keep] and [R, H] from ``select_pages``, for one query token a request.
    lse: fp32 [rows, heads], receives the log of the softmax sums.  workspace: device bytes for split work;
    allocated with the call where None, and then its own for as long as the prepared call lives (memory of the
    stream that is current then, on which other streams wait before its first launch there).
    """
    import torch

    L = lib()
    _inner(_bf16(q, "q"), "q"), _inner(_bf16(out, "out"), "out")
    rows, HQ, D = q.shape
    if out.shape != q.shape:
        raise ValueError("out must have q's shape")
    if k_cache.dim() != 4 or k_cache.shape != v_cache.shape or k_cache.dtype != v_cache.dtype:
        raise ValueError("k_cache and v_cache must be [pages, page_size, H, D] of one type")
    n_pages, page_size, H, Dc = k_cache.shape
    if Dc != D:
        raise ValueError("q and the caches must have one head size")
    eight = _is8(k_cache)
    if not eight:
        _bf16(k_cache, "k_cache")
    _inner(k_cache, "k_cache"), _inner(v_cache, "v_cache")
    R = kv_tokens.shape[0]
    n_queries, n_keys = _int(n_queries, "n_queries"), _int(n_keys, "n_keys")
    if q_base is None and R * n_queries > rows:
        raise ValueError(f"{R} requests of {n_queries} queries exceed the {rows} rows of q")
    for t, nm in ((kv_tokens, "kv_tokens"), (q_base, "q_base"), (q_tokens, "q_tokens")):
        _typed(t, torch.int32, nm, (R,))
    for t, nm in ((k_scale, "k_scale"), (v_scale, "v_scale")):
        _typed(t, torch.float32, nm, (n_pages, H), contiguous=False)
    _typed(lse, torch.float32, "lse", (rows, HQ), contiguous=False)
    _typed(status, torch.int32, "status")
    a = CAttendArgs()
    a.n_requests, a.n_q_heads, a.n_kv_heads, a.head_dim, a.n_queries, a.n_keys = R, HQ, H, D, n_queries, n_keys
    a.page_size, a.n_pool_pages = page_size, n_pages
    # selected pages are whatever sel holds: one past the rows of a view is not seen
    a.pt_stride = _table(page_table, R, n_keys if sel is None else 0, page_size)
    a.pt_pages = page_table.shape[1]
    a.cache_type = CACHE_E4M3 if eight else CACHE_BF16
    # a window past 32 bits holds every key there can be
    a.causal, a.window, a.n_splits = int(causal), _int(min(window, (1 << 31) - 1), "window"), _int(n_splits, "n_splits")
    a.scale = D ** -0.5 if scale is None else float(scale)
    a.q_tokens, a.q_base, a.kv_tokens, a.page_table = _ptr(q_tokens), _ptr(q_base), _ptr(kv_tokens), _ptr(page_table)
    a.q, a.out, a.lse = _ptr(q), _ptr(out), _ptr(lse)
    a.q_stride[0:2] = q.stride()[:2]
    a.out_stride[0:2] = out.stride()[:2]
    if lse is not None:
        a.lse_stride[:] = lse.stride()
    a.k_cache, a.v_cache, a.k_scale, a.v_scale = _ptr(k_cache), _ptr(v_cache), _ptr(k_scale), _ptr(v_scale)
    a.k_cache_stride[0:3] = k_cache.stride()[:3]
    a.v_cache_stride[0:3] = v_cache.stride()[:3]
    if k_scale is not None:
        a.k_scale_stride[:] = k_scale.stride()
    if v_scale is not None:
        a.v_scale_stride[:] = v_scale.stride()
    if sel is not None:
        keep = sel.shape[-1]
        _typed(sel, torch.int32, "sel", (R, H, keep))
        _typed(sel_count, torch.int32, "sel_count", (R, H))
        a.sel, a.sel_count, a.sel_stride = _ptr(sel), _ptr(sel_count), keep
    elif sel_count is not None:
        raise ValueError("sel_count without sel")
    a.status = _ptr(status)
    workspace = _workspace(a, L.kamera_attend_workspace(ctypes.byref(a)), workspace, q.device)
    _device(q, k_cache, v_cache, out, page_table, kv_tokens, q_base, q_tokens, k_scale, v_scale, sel, sel_count, lse,
            workspace, status)
    call = Prepared(L.kamera_attend_paged, a, (q, k_cache, v_cache, out, page_table, kv_tokens, q_base, q_tokens,
                                               k_scale, v_scale, sel, sel_count, lse, workspace, status))
    call.workspace = workspace
    return call


__all__ = ["STATUS_NO_PAGE", "STATUS_BAD_LENGTH", "MAX_REQUESTS", "MAX_SELECT_PAGES", "MAX_GROUP", "CACHE_BF16",
           "CACHE_E4M3", "CPageTablesArgs", "CAppendArgs", "CSelectArgs", "CAttendArgs", "Cache8", "page_tables",
           "prepare_page_tables", "append_paged8", "prepare_append_paged8", "select_pages", "prepare_select_pages",
           "attend_paged", "prepare_attend_paged", "attend_workspace"]
