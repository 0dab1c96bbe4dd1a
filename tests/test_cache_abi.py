"""The paged-cache entry points' host side, without a GPU: layouts, refusals,
workspace sizes, the binding's own checks, and the host layer under the CPU
sanitizers beside stand-in launches (tests/c/cache_stub.cpp)."""

from __future__ import annotations

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2606_23581_amd as km
from paper_2606_23581_amd import cache
from tests import cache_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_23581_amd", "csrc")
TC = os.path.join(ROOT, "tests", "c")

P = 0x10000000            # never dereferenced: validation looks at addresses only


def tables_args(**kw):
    a = km.CPageTablesArgs(n_requests=4, page_size=16, pt_stride=8, n_pool_pages=100, tokens_before=P,
                           tokens_after=P + 0x1000, free_pages=P + 0x2000, n_free=20, free_begin=P + 0x3000,
                           free_end=P + 0x3010, page_table=P + 0x4000, token_base=P + 0x5000, slots=P + 0x6000,
                           n_slots=64)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def strides(field, values):
    for i, v in enumerate(values):
        field[i] = v


def append_args(**kw):
    a = km.CAppendArgs(n_chunks=2, n_layers=3, n_heads=4, head_dim=128, n_tokens=40, page_size=16, pt_stride=4,
                       n_pool_pages=10, page_table=P, k=0x20000000, v=0x21000000, k_cache=0x30000000,
                       v_cache=0x31000000, k_scale=0x32000000, v_scale=0x33000000, k_sum=0x34000000,
                       k_sum_scale=0x35000000)
    for f in (a.k_stride, a.v_stride):
        strides(f, (3 * 40 * 512, 40 * 512, 512, 128))
    for f in (a.k_cache_stride, a.v_cache_stride):
        strides(f, (10 * 16 * 512, 16 * 512, 128, 16 * 128))
    for f in (a.k_scale_stride, a.v_scale_stride, a.k_sum_scale_stride):
        strides(f, (40, 4, 1))
    strides(a.k_sum_stride, (40 * 128, 512, 128))
    for k, v in kw.items():
        if isinstance(v, tuple):
            strides(getattr(a, k), v)
        else:
            setattr(a, k, v)
    return a


def select_args(**kw):
    a = km.CSelectArgs(n_requests=3, n_q_heads=8, n_kv_heads=2, head_dim=128, n_keys=1000, page_size=16, pt_stride=64,
                       n_pool_pages=200, kv_tokens=P, page_table=P + 0x1000, q=P + 0x10000, k_sum=0x20000000,
                       k_sum_scale=0x21000000, n_keep=8, n_first=1, n_last=1, sel=0x22000000, sel_count=0x23000000)
    strides(a.q_stride, (1024, 128))
    strides(a.k_sum_stride, (256, 128))
    strides(a.k_sum_scale_stride, (2, 1))
    for k, v in kw.items():
        if isinstance(v, tuple):
            strides(getattr(a, k), v)
        else:
            setattr(a, k, v)
    return a


def attend_args(**kw):
    a = km.CAttendArgs(n_requests=2, n_q_heads=16, n_kv_heads=2, head_dim=128, n_queries=1, n_keys=4096, page_size=16,
                       pt_stride=256, n_pool_pages=600, cache_type=1, causal=1, scale=0.1, kv_tokens=P,
                       page_table=P + 0x1000, q=0x20000000, out=0x21000000, k_cache=0x30000000, v_cache=0x40000000,
                       k_scale=0x50000000, v_scale=0x51000000, workspace=0x60000000, workspace_bytes=1 << 30)
    strides(a.q_stride, (2048, 128))
    strides(a.out_stride, (2048, 128))
    strides(a.lse_stride, (16, 1))
    for f in (a.k_cache_stride, a.v_cache_stride):
        strides(f, (2 * 16 * 128, 128, 16 * 128))
    for f in (a.k_scale_stride, a.v_scale_stride):
        strides(f, (2, 1))
    for k, v in kw.items():
        if isinstance(v, tuple):
            strides(getattr(a, k), v)
        else:
            setattr(a, k, v)
    return a


MAKE = (tables_args, append_args, select_args, attend_args)

CASES = [
    (0, {}, km.OK),
    (0, dict(n_requests=0, tokens_after=None, page_table=None), km.OK),
    (0, dict(tokens_before=None, free_begin=None, slots=None, n_slots=0), km.OK),
    (0, dict(n_requests=-1), km.ERR_SHAPE),
    (0, dict(n_requests=8193), km.ERR_RANGE),
    (0, dict(page_size=0), km.ERR_SHAPE),
    (0, dict(pt_stride=0), km.ERR_SHAPE),
    (0, dict(n_pool_pages=0), km.ERR_SHAPE),
    (0, dict(pt_stride=1 << 28), km.ERR_RANGE),
    (0, dict(n_slots=1 << 60), km.ERR_RANGE),
    (0, dict(tokens_after=None), km.ERR_NULL),
    (0, dict(page_table=None), km.ERR_NULL),
    (0, dict(token_base=None), km.ERR_NULL),
    (0, dict(free_end=None), km.ERR_NULL),
    (0, dict(free_pages=None), km.ERR_NULL),
    (0, dict(free_pages=None, n_free=0), km.OK),
    (0, dict(slots=None), km.ERR_NULL),
    (0, dict(free_end=P + 0x3000), km.ERR_ALIAS),
    (0, dict(token_base=P + 0xFFC), km.ERR_ALIAS),
    (0, dict(slots=P + 0x2000 + 76), km.ERR_ALIAS),
    (0, dict(slots=P + 0x4000 + 4 * 31), km.ERR_ALIAS),
    (1, {}, km.OK),
    (1, dict(k_sum=None, k_sum_scale=None), km.OK),
    (1, dict(n_tokens=0, k=None), km.OK),
    (1, dict(head_dim=96), km.ERR_UNSUPPORTED),
    (1, dict(page_size=48), km.ERR_UNSUPPORTED),
    (1, dict(page_size=128), km.ERR_UNSUPPORTED),
    (1, dict(n_layers=-1), km.ERR_SHAPE),
    (1, dict(pt_stride=2), km.ERR_SHAPE),
    (1, dict(n_pool_pages=0), km.ERR_SHAPE),
    (1, dict(page_table=None), km.ERR_NULL),
    (1, dict(v=None), km.ERR_NULL),
    (1, dict(k_scale=None), km.ERR_NULL),
    (1, dict(k_sum=None), km.ERR_NULL),
    (1, dict(k_sum_scale=None), km.ERR_NULL),
    (1, dict(k=0x20000008), km.ERR_ALIGN),
    (1, dict(v_stride=(3 * 40 * 512, 40 * 512, 516, 128)), km.ERR_ALIGN),
    (1, dict(v_cache=0x31000008), km.ERR_ALIGN),
    (1, dict(k_cache_stride=(10 * 16 * 512, 16 * 512, 136, 16 * 128)), km.ERR_ALIGN),
    (1, dict(k_sum_stride=(40 * 128, 512, 120)), km.ERR_ALIGN),
    (1, dict(n_chunks=1 << 26, n_heads=32), km.ERR_RANGE),
    (1, dict(k_cache_stride=(-(1 << 62), 16 * 512, 128, 16 * 128)), km.ERR_RANGE),
    (1, dict(k_cache=0x20000000), km.ERR_ALIAS),
    (1, dict(v_cache=0x30000000), km.ERR_ALIAS),
    (1, dict(k_sum=0x20000100), km.ERR_ALIAS),
    (2, {}, km.OK),
    (2, dict(n_requests=0, q=None), km.OK),
    (2, dict(head_dim=80), km.ERR_UNSUPPORTED),
    (2, dict(n_q_heads=9), km.ERR_SHAPE),
    (2, dict(n_kv_heads=0), km.ERR_SHAPE),
    (2, dict(n_q_heads=130), km.ERR_RANGE),
    (2, dict(page_size=24), km.ERR_UNSUPPORTED),
    (2, dict(n_last=0), km.ERR_SHAPE),
    (2, dict(n_first=8), km.ERR_SHAPE),
    (2, dict(n_first=-1), km.ERR_SHAPE),
    (2, dict(n_keys=16 * 32768 + 1, pt_stride=40000), km.ERR_RANGE),
    (2, dict(pt_stride=62), km.ERR_SHAPE),
    (2, dict(sel=None), km.ERR_NULL),
    (2, dict(k_sum_scale=None), km.ERR_NULL),
    (2, dict(k_sum=0x20000004), km.ERR_ALIGN),
    (2, dict(sel=P + 0x10000), km.ERR_ALIAS),
    (2, dict(sel_count=0x22000000), km.ERR_ALIAS),
    (2, dict(sel=P + 0x1000), km.ERR_ALIAS),
    (2, dict(n_requests=1 << 22), km.ERR_RANGE),
    (3, {}, km.OK),
    (3, dict(n_requests=0, q=None), km.OK),
    (3, dict(n_queries=0, q=None), km.OK),
    (3, dict(cache_type=0, k_scale=None, v_scale=None), km.OK),
    (3, dict(head_dim=256), km.ERR_UNSUPPORTED),
    (3, dict(n_q_heads=15), km.ERR_SHAPE),
    (3, dict(n_q_heads=130), km.ERR_RANGE),
    (3, dict(page_size=24), km.ERR_UNSUPPORTED),
    (3, dict(cache_type=2), km.ERR_SHAPE),
    (3, dict(causal=2), km.ERR_SHAPE),
    (3, dict(window=-1), km.ERR_SHAPE),
    (3, dict(window=5, causal=0), km.ERR_SHAPE),
    (3, dict(scale=float("nan")), km.ERR_SHAPE),
    (3, dict(n_splits=513), km.ERR_SHAPE),
    (3, dict(n_keys=2147483647, pt_stride=1 << 28), km.ERR_RANGE),
    (3, dict(pt_stride=255), km.ERR_SHAPE),
    (3, dict(page_table=None), km.ERR_NULL),
    (3, dict(out=None), km.ERR_NULL),
    (3, dict(kv_tokens=None), km.ERR_NULL),
    (3, dict(v_scale=None), km.ERR_NULL),
    (3, dict(sel=P), km.ERR_NULL),
    (3, dict(sel=P, sel_count=P, sel_stride=8), km.OK),
    (3, dict(sel=P, sel_count=P, sel_stride=8, n_queries=2), km.ERR_UNSUPPORTED),
    (3, dict(q=0x20000002), km.ERR_ALIGN),
    (3, dict(out_stride=(2048, 132)), km.ERR_ALIGN),
    (3, dict(k_cache_stride=(2 * 16 * 128, 120, 16 * 128)), km.ERR_ALIGN),
    (3, dict(v_cache_stride=(2 * 16 * 128, 1 << 25, 16 * 128)), km.ERR_RANGE),
    (3, dict(workspace=None), km.ERR_NULL),
    (3, dict(workspace_bytes=100), km.ERR_SHAPE),
    (3, dict(workspace=0x60000008), km.ERR_ALIGN),
    (3, dict(workspace=None, n_splits=1), km.OK),
    (3, dict(out=0x20000000), km.ERR_ALIAS),
    (3, dict(out=0x30000000), km.ERR_ALIAS),
    (3, dict(workspace=0x21000000), km.ERR_ALIAS),
    (3, dict(lse=0x21000000), km.ERR_ALIAS),
    (3, dict(n_requests=1 << 28, n_splits=1), km.ERR_RANGE),
    # 2^25 rows of long prompts in one part each; joined parts of as many are past one launch
    (3, dict(n_queries=1 << 20, out=0x2000000000, k_cache=0x4000000000, v_cache=0x5000000000), km.OK),
    (3, dict(n_queries=1 << 20, out=0x2000000000, k_cache=0x4000000000, v_cache=0x5000000000, n_splits=2), km.ERR_RANGE),
]


@pytest.mark.parametrize("which,change,code", CASES)
def test_validation(which, change, code):
    a = MAKE[which](**change)
    assert km.lib().kamera_validate_cache(which, ctypes.byref(a)) == code, km.last_error()
    assert (km.last_error() == "") == (code == km.OK)


@pytest.mark.parametrize("page_size,units_a_workgroup", [(16, 4), (32, 2), (64, 1)])
def test_append_fits_one_launch(page_size, units_a_workgroup):
    """A page of 64 tokens takes the four waves of a workgroup, one of 16 tokens one of them: a launch has at most
    2^32 - 1 work-items, 256 a workgroup.  One token a chunk, one head: two units a chunk (keys, values)."""
    most = ((1 << 32) - 1) // 256 * units_a_workgroup // 2
    for n, code in ((most, km.OK), (most + 1, km.ERR_RANGE)):
        a = append_args(n_chunks=n, n_layers=1, n_heads=1, n_tokens=1, page_size=page_size, k_stride=(0,), v_stride=(0,))
        assert km.lib().kamera_validate_cache(1, ctypes.byref(a)) == code, km.last_error()
    # a batch of ragged prompts of which only the longest is known on the host
    a = append_args(n_chunks=256, n_layers=80, n_heads=8, n_tokens=8192, page_size=page_size, pt_stride=512)
    for f in (a.k_stride, a.v_stride, a.k_cache_stride, a.v_cache_stride):
        strides(f, (0, 0))
    assert km.lib().kamera_validate_cache(1, ctypes.byref(a)) == km.ERR_RANGE


def test_validation_of_nothing():
    L = km.lib()
    for which in range(4):
        assert L.kamera_validate_cache(which, None) == km.ERR_NULL
    assert L.kamera_validate_cache(4, None) == km.ERR_SHAPE
    assert L.kamera_attend_workspace(None) == km.ERR_NULL


def test_struct_layout():
    L = km.lib()
    for which, cls in ((6, km.CPageTablesArgs), (7, km.CAppendArgs), (8, km.CSelectArgs), (9, km.CAttendArgs)):
        assert L.kamera_struct_size(which) == ctypes.sizeof(cls)


def test_workspace():
    L = km.lib()
    a = attend_args()
    a.n_splits = 5
    # every (request, query head, query) row, its parts: D sums, and four words for the maximum and sums
    assert L.kamera_attend_workspace(ctypes.byref(a)) == 2 * 16 * 5 * (128 + 4) * 4
    a.n_splits = 1
    assert L.kamera_attend_workspace(ctypes.byref(a)) == 0
    a.n_splits, a.n_keys = 0, 200
    assert L.kamera_attend_workspace(ctypes.byref(a)) == 0
    a.n_keys, a.n_requests = 4096, 1000
    assert L.kamera_attend_workspace(ctypes.byref(a)) == 0
    a.head_dim = 100
    assert L.kamera_attend_workspace(ctypes.byref(a)) == km.ERR_UNSUPPORTED


def test_binding_refuses():
    """Types, shapes and layouts that the binding itself turns down, on CPU tensors."""
    bf, i4 = torch.bfloat16, torch.int32
    q = torch.zeros((2, 8, 128), dtype=bf)
    cache = torch.zeros((4, 16, 2, 128), dtype=torch.uint8)
    scale = torch.ones((4, 2))
    table, kv = torch.zeros((2, 2), dtype=i4), torch.zeros(2, dtype=i4)

    def attend(**kw):
        a = dict(q=q, k_cache=cache, v_cache=cache.clone(), out=torch.zeros_like(q), page_table=table, kv_tokens=kv,
                 n_queries=1, n_keys=32, k_scale=scale, v_scale=scale)
        a.update(kw)
        km.prepare_attend_paged(**a)

    with pytest.raises(ValueError, match="device memory"):
        attend()
    for bad, err in ((dict(q=q.float()), TypeError), (dict(out=q[:1]), ValueError),
                     (dict(k_cache=cache.to(bf)), ValueError), (dict(kv_tokens=kv.long()), TypeError),
                     (dict(page_table=table[:1]), ValueError), (dict(page_table=table.t()), ValueError),
                     (dict(k_scale=scale.double()), TypeError), (dict(k_scale=scale[:3]), ValueError),
                     (dict(n_queries=2), ValueError), (dict(sel_count=kv), ValueError),
                     (dict(sel=torch.zeros((2, 3, 4), dtype=i4)), ValueError),
                     (dict(lse=torch.zeros(2, 8, dtype=bf)), TypeError), (dict(window=-2), km.KameraError),
                     (dict(n_keys=-1), km.KameraError)):
        with pytest.raises(err):
            attend(**bad)
    with pytest.raises(TypeError):
        km.prepare_append_paged8(q[None, None].float(), q[None, None], cache[None], cache[None], scale[None],
                                 scale[None], table)
    with pytest.raises(ValueError):
        km.prepare_append_paged8(q[None, None], q[None, None], cache[None], cache[None], scale[None], scale[None],
                                 table[:1], row_base=kv[:1])
    with pytest.raises(ValueError):
        km.prepare_page_tables(kv, kv, kv, table[:1], page_size=16, n_pool_pages=4, free_end=kv[:1],
                               token_base=torch.zeros(3, dtype=i4))
    with pytest.raises(TypeError):
        km.prepare_select_pages(q, cache[:, 0], scale, table, kv, torch.zeros((2, 2, 4), dtype=i4),
                                torch.zeros((2, 2), dtype=i4), n_keys=32, page_size=16)


def test_binding_takes_views_of_page_tables():
    """Rows with a stride: what a call may look up has to be there."""
    i4 = torch.int32
    whole = torch.zeros((3, 20), dtype=i4)
    for view, tokens, ok in ((whole, None, True), (whole[:, :8], 128, True), (whole[:, 12:], 128, True),
                             (whole[:, 12:], 129, False), (whole[:, :8], 129, False), (whole[:, :8], None, True),
                             (whole[:, 12:], None, False), (whole[1:, 12:], None, False), (whole[:2, 12:], None, True),
                             (whole[:1, 12:], None, True)):
        n = view.shape[0]
        if ok:
            assert cache._table(view, n, tokens, 16) == (20 if n > 1 else view.shape[1])
        else:
            with pytest.raises(ValueError):
                cache._table(view, n, tokens, 16)


@pytest.mark.parametrize("which,change,code", [
    (1, dict(pt_stride=20, pt_pages=3), km.OK),
    (1, dict(pt_stride=20, pt_pages=2), km.ERR_SHAPE),
    (1, dict(pt_stride=20, pt_pages=-1), km.ERR_SHAPE),
    (3, dict(pt_stride=500, pt_pages=256), km.OK),
    (3, dict(pt_stride=500, pt_pages=255), km.ERR_SHAPE),
    (3, dict(pt_stride=500, pt_pages=-1), km.ERR_SHAPE),
    # selected pages are whatever sel holds
    (3, dict(pt_stride=500, pt_pages=8, sel=P, sel_count=P, sel_stride=8), km.OK),
    # the last row ends with its own pages: what lies behind them is not the table's
    (1, dict(pt_stride=20, pt_pages=3, page_table=0x30000000 - 4 * 23), km.OK),
    (3, dict(pt_stride=500, pt_pages=256, page_table=0x21000000 - 4 * 756), km.OK),
])
def test_rows_of_a_page_table_narrower_than_their_stride(which, change, code):
    a = MAKE[which](**change)
    assert km.lib().kamera_validate_cache(which, ctypes.byref(a)) == code, km.last_error()


@pytest.mark.parametrize("which,change", [
    # attention: out, lse or the workspace over any of the arrays that a call reads
    (3, dict(kv_tokens=0x21000000)),
    (3, dict(q_tokens=0x21000000 + 2 * 2 * 2048 - 4)),
    (3, dict(q_base=0x21000000 + 4)),
    (3, dict(lse=P + 4)),
    (3, dict(workspace=P)),
    (3, dict(q_tokens=0x60000000)),
    (3, dict(sel=0x21000000 - 4 * 31, sel_count=P, sel_stride=8)),
    (3, dict(sel=P, sel_count=0x21000000 - 4 * 3, sel_stride=8)),
    # append: caches, scales or sums over the table or the lengths
    (1, dict(page_table=0x30000000 - 4 * 7)),
    (1, dict(chunk_tokens=0x31000000)),
    (1, dict(tokens_before=0x32000000 + 4)),
    (1, dict(row_base=0x34000000 - 4)),
    (1, dict(page_table=0x35000000)),
])
def test_outputs_over_inputs_are_refused(which, change):
    a = MAKE[which](**change)
    assert km.lib().kamera_validate_cache(which, ctypes.byref(a)) == km.ERR_ALIAS, km.last_error()


@pytest.mark.parametrize("which,change", [
    (3, dict(q_tokens=0x21000000 - 8)),
    (3, dict(sel=0x21000000 - 4 * 32, sel_count=0x21000000 + 2 * 2 * 2048, sel_stride=8)),
    (3, dict(kv_tokens=P, q_tokens=P, q_base=P)),
    (1, dict(page_table=0x30000000 - 4 * 8, chunk_tokens=0x34000000 - 8, tokens_before=0x34000000 - 8)),
])
def test_outputs_beside_inputs_are_taken(which, change):
    a = MAKE[which](**change)
    assert km.lib().kamera_validate_cache(which, ctypes.byref(a)) == km.OK, km.last_error()


def test_views_of_page_tables_end_where_the_view_does(monkeypatch):
    """A call is told the pages of its view, not those of the tensor behind it."""
    monkeypatch.setattr(cache, "_device", lambda *t: None)
    whole = torch.zeros((3, 20), dtype=torch.int32)
    rows = torch.zeros((3, 1, 24, 2, 128), dtype=torch.bfloat16)
    planes = [torch.zeros((1, 4, 16, 2, 128), dtype=torch.uint8) for _ in range(2)]
    scales = [torch.ones((1, 4, 2)) for _ in range(2)]
    q = torch.zeros((3, 8, 128), dtype=torch.bfloat16)
    kv, sel = torch.zeros(3, dtype=torch.int32), torch.zeros((3, 2, 2), dtype=torch.int32)
    for view in (whole[:, :2], whole[:, 18:], whole[:, 5:9], whole):
        a = km.prepare_append_paged8(rows, rows, *planes, *scales, view).args
        assert (a.pt_stride, a.pt_pages) == (20, view.shape[1])
        for kw in (dict(sel=sel, sel_count=sel[:, :, 0].contiguous()), {}):
            a = km.prepare_attend_paged(q, planes[0][0], planes[1][0], torch.zeros_like(q), view, kv, n_queries=1,
                                        n_keys=32, k_scale=scales[0][0], v_scale=scales[1][0], **kw).args
            assert (a.pt_stride, a.pt_pages) == (20, view.shape[1])


def test_a_given_workspace_is_as_long_as_it_says(monkeypatch):
    """A view's elements may be many more than the memory behind it holds, or lie apart."""
    monkeypatch.setattr(cache, "_device", lambda *t: None)
    q, kv = torch.zeros((2, 8, 128), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    planes = [torch.zeros((4, 16, 2, 128), dtype=torch.uint8) for _ in range(2)]
    scale, table = torch.ones((4, 2)), torch.zeros((2, 300), dtype=torch.int32)

    def attend(workspace):
        return km.prepare_attend_paged(q, *planes, torch.zeros_like(q), table, kv, n_queries=1, n_keys=4096,
                                       k_scale=scale, v_scale=scale, n_splits=4, workspace=workspace)

    def select(workspace):
        return km.prepare_select_pages(q, torch.zeros((4, 2, 128), dtype=torch.int8), scale,
                                       torch.zeros((2, 3000), dtype=torch.int32), kv,
                                       torch.zeros((2, 2, 4), dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32),
                                       n_keys=40000, page_size=16, workspace=workspace)

    for call in (attend, select):
        need = call(None).args.workspace_bytes
        assert need > 0
        assert call(torch.zeros(need // 4)).args.workspace_bytes == need
        for bad in (torch.zeros(16).expand(need, 16), torch.zeros(1).expand(need), torch.zeros((need, 2))[:, 0]):
            with pytest.raises(ValueError, match="contiguous"):
                call(bad)


def test_numbers_past_32_bits(monkeypatch):
    """They would reach the library as their low 32 bits, 2^32 + 5 keys as 5: refused, but for a window, which then
    holds every key."""
    monkeypatch.setattr(cache, "_device", lambda *t: None)
    i4 = torch.int32
    q, kv, table = torch.zeros((2, 8, 128), dtype=torch.bfloat16), torch.zeros(2, dtype=i4), torch.zeros((2, 3), dtype=i4)
    planes = [torch.zeros((4, 16, 2, 128), dtype=torch.uint8) for _ in range(2)]
    scale, rows = torch.ones((4, 2)), torch.zeros((1, 30, 2, 128), dtype=torch.bfloat16)

    def attend(**kw):
        a = dict(n_queries=1, n_keys=48, q_base=kv, k_scale=scale, v_scale=scale)
        return km.prepare_attend_paged(q, *planes, torch.zeros_like(q), table, kv, **dict(a, **kw))

    def select(**kw):
        a = dict(n_keys=48, page_size=16)
        km.prepare_select_pages(q, torch.zeros((4, 2, 128), dtype=torch.int8), scale, table, kv,
                                torch.zeros((2, 2, 4), dtype=i4), torch.zeros((2, 2), dtype=i4), **dict(a, **kw))

    def append(**kw):
        a = dict(n_tokens=20, row_base=kv)
        km.prepare_append_paged8(rows, rows, *[p[None] for p in planes], *[scale[None].clone() for _ in range(2)], table,
                                 **dict(a, **kw))

    def tables(**kw):
        a = dict(page_size=16, n_pool_pages=4, free_end=torch.zeros(1, dtype=i4), token_base=torch.zeros(3, dtype=i4))
        km.prepare_page_tables(None, kv, torch.zeros(5, dtype=i4), table, **dict(a, **kw))

    far = 1 << 32
    for call, names in ((attend, ("n_keys", "n_queries", "n_splits")),
                        (select, ("n_keys", "page_size", "n_first", "n_last")), (append, ("n_tokens",)),
                        (tables, ("page_size", "n_pool_pages"))):
        call()
        for name in names:
            for x in (far + 1, far + 16, -far + 1, 1 << 31):
                with pytest.raises(ValueError, match=name):
                    call(**{name: x})
    assert attend(window=far + 5).args.window == (1 << 31) - 1
    with pytest.raises(ValueError, match="window"):
        attend(window=-far + 5)


def test_reference_e4m3_agrees_with_torch():
    """The tests' own e4m3 rounding against torch's cast, at every value, midpoint and many others."""
    pos = ref.e4m3_values()[:127]
    x = np.concatenate([pos, (pos[1:] + pos[:-1]) / 2, -pos, np.random.default_rng(0).standard_normal(20000) * 3,
                        np.random.default_rng(1).standard_normal(20000) * 0.01]).astype(np.float32)
    want = torch.tensor(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(ref.encode(x.astype(np.float64)), want)


def test_no_more_of_a_table_is_looked_up_than_there_is(tmp_path):
    _host_program(tmp_path, "cache_params", [], ("launch_stub.cpp", "cache_params.cpp"))


def _host_program(tmp_path, name, flags, sources):
    if shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("no g++ or HIP headers")
    exe = str(tmp_path / name)
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I",
           os.path.join(ROOT, "include"), "-I", CSRC, "-I", TC, *flags,
           *[os.path.join(CSRC, f) for f in ("kamera_abi.cpp", "kamera_cache.cpp")],
           *[os.path.join(TC, f) for f in sources], "-o", exe, "-pthread"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), (r.stdout[-2000:], r.stderr[-4000:])


def _sanitized(tmp_path, name, flags):
    if shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("no g++ or HIP headers")
    exe = str(tmp_path / name)
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-D__HIP_PLATFORM_AMD__", "-I",
           "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", TC, *flags,
           *[os.path.join(CSRC, f) for f in ("kamera_abi.cpp", "kamera_cache.cpp")],
           *[os.path.join(TC, f) for f in ("launch_stub.cpp", "cache_stub.cpp", "cache_sanitize.cpp")], "-o", exe,
           "-pthread"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300,
                       env=dict(os.environ, UBSAN_OPTIONS="print_stacktrace=1", TSAN_OPTIONS="halt_on_error=1"))
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), (r.stdout[-2000:], r.stderr[-4000:])


def test_host_layer_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    _sanitized(tmp_path, "cache_asan", ["-fsanitize=address,undefined", "-fno-sanitize-recover=undefined"])


def test_host_layer_under_thread_sanitizer(tmp_path):
    _sanitized(tmp_path, "cache_tsan", ["-fsanitize=thread"])
