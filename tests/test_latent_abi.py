"""The latent-cache entry points' host side, without a GPU: layouts, refusals,
workspace sizes, the binding's own checks, and the host layer under the CPU
sanitizers beside stand-in launches (tests/c/latent_stub.cpp)."""

from __future__ import annotations

import ctypes
import math
import os
import random
import shutil
import subprocess

import pytest
import torch

import paper_2606_23581_amd as km
from paper_2606_23581_amd import latent
from tests import latent_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_23581_amd", "csrc")
TC = os.path.join(ROOT, "tests", "c")

P = 0x10000000            # never dereferenced: validation looks at addresses only


def fill(a, kw):
    for k, v in kw.items():
        if isinstance(v, tuple):
            for i, x in enumerate(v):
                getattr(a, k)[i] = x
        elif "." in k:
            setattr(getattr(a, k.split(".")[0]), k.split(".")[1], v)
        else:
            setattr(a, k, v)
    return a


def rotate_args(**kw):
    a = km.CAppendRotatedArgs(n_chunks=2, n_layers=3, n_tokens=40, n_k_heads=4, k_dim=128, n_v_heads=4, v_dim=128,
                              n_q_heads=8, page_size=16, pt_stride=4, n_pool_pages=10, page_table=P, k=0x20000000,
                              v=0x21000000, q=0x22000000, q_out=0x23000000, k_cache=0x30000000, v_cache=0x31000000)
    a.rope = km.RopeSpec(theta=1e4, rope_dim=64).to_c()
    fill(a, dict(k_stride=(3 * 40 * 512, 40 * 512, 512, 128), v_stride=(3 * 40 * 512, 40 * 512, 512, 128),
                 q_stride=(3 * 40 * 1024, 40 * 1024, 1024, 128), q_out_stride=(3 * 40 * 512, 40 * 512, 512, 64),
                 k_cache_stride=(81920, 8192, 512, 128), v_cache_stride=(81920, 8192, 512, 128)))
    return fill(a, kw)


def project_args(**kw):
    a = km.CProjectArgs(n_rows=100, n_heads=16, n_in=128, n_out=512, x=0x20000000, w=0x21000000, out=0x22000000)
    fill(a, dict(x_stride=(16 * 128, 128), w_stride=(128 * 512, 512, 1), out_stride=(16 * 512, 512)))
    return fill(a, kw)


def expand_args(**kw):
    a = km.CExpandArgs(n_requests=3, n_heads=16, n_in=512, n_out=256, n_keys=1000, page_size=16, pt_stride=64,
                       n_pool_pages=200, kv_tokens=P, page_table=P + 0x1000, cache=0x20000000, w=0x21000000, out=0x22000000)
    fill(a, dict(cache_stride=(16 * 576, 576), w_stride=(512 * 256, 1, 512), out_stride=(16 * 256, 256)))
    return fill(a, kw)


def latent_args(**kw):
    a = km.CAttendLatentArgs(n_requests=2, n_heads=16, latent_dim=512, rope_dim=64, n_queries=1, n_keys=4096, page_size=16,
                             pt_stride=256, n_pool_pages=600, causal=1, scale=0.1, kv_tokens=P, page_table=P + 0x1000,
                             q=0x20000000, out=0x21000000, cache=0x30000000, workspace=0x60000000, workspace_bytes=1 << 30)
    fill(a, dict(q_stride=(16 * 576, 576), out_stride=(16 * 512, 512), lse_stride=(16, 1), cache_stride=(16 * 576, 576)))
    return fill(a, kw)


def expanded_args(**kw):
    a = km.CAttendExpandedArgs(n_requests=2, n_heads=16, head_dim=128, rope_dim=64, n_queries=100, n_keys=4096, page_size=16,
                               pt_stride=256, n_pool_pages=600, causal=1, scale=0.1, kv_tokens=P, page_table=P + 0x1000,
                               q=0x20000000, out=0x21000000, k=0x40000000, v=0x48000000, rope_cache=0x30000000,
                               workspace=0x60000000, workspace_bytes=1 << 30)
    fill(a, dict(q_stride=(16 * 192, 192), out_stride=(16 * 128, 128), lse_stride=(16, 1), k_stride=(16 * 128, 128),
                 v_stride=(16 * 128, 128), rope_cache_stride=(16 * 576, 576)))
    return fill(a, kw)


MAKE = (rotate_args, project_args, expand_args, latent_args, expanded_args)
NEOX8 = km.RopeSpec(theta=1e4, rope_dim=8).to_c()

CASES = [
    (0, {}, km.OK),
    (0, dict(n_chunks=0, k=None), km.OK),
    (0, dict(n_tokens=0, page_table=None), km.OK),
    (0, dict(v=None, v_cache=None), km.OK),
    (0, dict(q=None, q_out=None), km.OK),
    (0, dict(n_k_heads=0, n_v_heads=0, n_q_heads=0), km.OK),
    (0, dict(n_layers=-1), km.ERR_SHAPE),
    (0, dict(n_q_heads=-1), km.ERR_SHAPE),
    (0, dict(k_dim=100), km.ERR_SHAPE),
    (0, dict(v_dim=0), km.ERR_SHAPE),
    (0, dict(k_dim=4104), km.ERR_RANGE),
    (0, {"rope.rope_dim": 130}, km.ERR_RANGE),
    (0, {"rope.rope_offset": 72}, km.ERR_SHAPE),
    (0, {"rope.rope_offset": 4}, km.ERR_UNSUPPORTED),
    (0, dict(rope=NEOX8), km.ERR_UNSUPPORTED),
    (0, {"rope.theta": -1.0}, km.ERR_SHAPE),
    (0, {"rope.n_sections": 3}, km.ERR_SHAPE),
    (0, {"scaling.kind": 4}, km.ERR_SHAPE),
    (0, {"scaling.kind": 1}, km.ERR_SHAPE),
    (0, {"scaling.kind": 1, "scaling.factor": 2.0}, km.OK),
    (0, {"scaling.kind": 1, "scaling.factor": 2.0, "scaling.amplitude": float("inf")}, km.ERR_SHAPE),
    (0, {"scaling.kind": 2, "scaling.factor": 2.0}, km.ERR_SHAPE),
    (0, {"scaling.kind": 2, "scaling.factor": 2.0, "scaling.original_tokens": 100.0, "scaling.low_turns": 1.0,
         "scaling.high_turns": 1.0}, km.ERR_SHAPE),
    (0, {"scaling.kind": 3, "scaling.factor": 2.0, "scaling.original_tokens": 100.0, "scaling.low_turns": 1.0,
         "scaling.high_turns": 2.0}, km.OK),
    (0, {"scaling.kind": 3, "scaling.factor": 2.0, "scaling.original_tokens": 100.0, "scaling.low_turns": 1.0,
         "scaling.high_turns": 2.0, "rope.theta": 1.0}, km.ERR_SHAPE),
    (0, dict(page_size=0), km.ERR_SHAPE),
    (0, dict(n_pool_pages=0), km.ERR_SHAPE),
    (0, dict(pt_pages=-1), km.ERR_SHAPE),
    (0, dict(page_table=None), km.ERR_NULL),
    (0, dict(k=None), km.ERR_NULL),
    (0, dict(k_cache=None), km.ERR_NULL),
    (0, dict(v_cache=None), km.ERR_NULL),
    (0, dict(q_out=None), km.ERR_NULL),
    (0, dict(k=0x20000008), km.ERR_ALIGN),
    (0, dict(q_out_stride=(0, 0, 516, 64)), km.ERR_ALIGN),
    (0, dict(v_cache_stride=(81920, 8192, 516, 128)), km.ERR_ALIGN),
    (0, dict(n_chunks=1 << 29), km.ERR_ALIAS),
    (0, dict(n_layers=1 << 28, k_stride=(0, 0), v_stride=(0, 0), q_stride=(0, 0), q_out_stride=(0, 0), k_cache_stride=(0,),
             v_cache_stride=(0,)), km.ERR_RANGE),
    (0, dict(n_k_heads=1 << 20), km.ERR_RANGE),
    (0, dict(k_cache_stride=(-(1 << 62), 8192, 512, 128)), km.ERR_RANGE),
    (0, dict(k_cache=0x20000000), km.ERR_ALIAS),
    (0, dict(v_cache=0x30000000), km.ERR_ALIAS),
    (0, dict(q_out=0x30000000), km.ERR_ALIAS),
    (0, dict(q_out=0x22000000), km.ERR_ALIAS),
    (0, dict(chunk_tokens=0x23000000), km.ERR_ALIAS),
    (0, dict(positions=0x31000000), km.ERR_ALIAS),
    # queries in place, with the same strides
    (0, dict(q_out=0x22000000, q_out_stride=(3 * 40 * 1024, 40 * 1024, 1024, 128)), km.OK),
    (0, dict(q_out=0x22000010, q_out_stride=(3 * 40 * 1024, 40 * 1024, 1024, 128)), km.ERR_ALIAS),
    # ... and keys beside them in one tensor
    (0, dict(k=0x22000000 + 2048, k_stride=(3 * 40 * 2048, 40 * 2048, 2048, 128), q_out=0x22000000,
             q_stride=(3 * 40 * 2048, 40 * 2048, 2048, 128), q_out_stride=(3 * 40 * 2048, 40 * 2048, 2048, 128)), km.OK),
    (0, dict(k=0x22000000 + 1024, k_stride=(3 * 40 * 2048, 40 * 2048, 2048, 128), q_out=0x22000000,
             q_stride=(3 * 40 * 2048, 40 * 2048, 2048, 128), q_out_stride=(3 * 40 * 2048, 40 * 2048, 2048, 128)), km.ERR_ALIAS),
    # keys and values of a token, of a page, beside each other
    (0, dict(v_cache=0x30000000 + 1024, k_cache_stride=(163840, 16384, 1024, 128), v_cache_stride=(163840, 16384, 1024, 128)),
     km.OK),
    (0, dict(v_cache=0x30000000 + 1008, k_cache_stride=(163840, 16384, 1024, 128), v_cache_stride=(163840, 16384, 1024, 128)),
     km.ERR_ALIAS),
    (0, dict(v_cache=0x30000000 + 16384, k_cache_stride=(163840, 16384, 128, 2048), v_cache_stride=(163840, 16384, 128, 2048)),
     km.OK),
    (1, {}, km.OK),
    (1, dict(n_rows=0, x=None), km.OK),
    (1, dict(n_heads=0, w=None), km.OK),
    (1, dict(n_rows=-1), km.ERR_SHAPE),
    (1, dict(n_heads=-1), km.ERR_SHAPE),
    (1, dict(n_in=96), km.ERR_UNSUPPORTED),
    (1, dict(n_out=0), km.ERR_UNSUPPORTED),
    (1, dict(n_out=4160), km.ERR_RANGE),
    (1, dict(x=None), km.ERR_NULL),
    (1, dict(w=None), km.ERR_NULL),
    (1, dict(out=None), km.ERR_NULL),
    (1, dict(w_stride=(128 * 512, 1, 128)), km.OK),
    (1, dict(w_stride=(128 * 512, 1, 132)), km.ERR_ALIGN),
    (1, dict(w_stride=(128 * 512, 2, 256)), km.ERR_ALIGN),
    (1, dict(x_stride=(16 * 128, 124)), km.ERR_ALIGN),
    (1, dict(out=0x22000008), km.ERR_ALIGN),
    (1, dict(x_stride=(128, 0), w_stride=(0, 512, 1)), km.OK),
    (1, dict(out=0x20000000), km.ERR_ALIAS),
    (1, dict(out=0x21000000), km.ERR_ALIAS),
    # columns of one tensor
    (1, dict(out=0x20000000 + 256, x_stride=(16 * 640, 640), out_stride=(16 * 640, 640)), km.OK),
    (1, dict(out=0x20000000 + 240, x_stride=(16 * 640, 640), out_stride=(16 * 640, 640)), km.ERR_ALIAS),
    (1, dict(n_rows=2147483647, n_heads=4096), km.ERR_RANGE),
    (1, dict(x_stride=(1 << 62, 128)), km.ERR_RANGE),
    (2, {}, km.OK),
    (2, dict(n_requests=0, cache=None), km.OK),
    (2, dict(n_keys=0, page_table=None), km.OK),
    (2, dict(n_keys=-1), km.ERR_SHAPE),
    (2, dict(page_size=0), km.ERR_SHAPE),
    (2, dict(n_in=500), km.ERR_UNSUPPORTED),
    (2, dict(pt_stride=62), km.ERR_SHAPE),
    (2, dict(kv_tokens=None), km.ERR_NULL),
    (2, dict(cache=None), km.ERR_NULL),
    (2, dict(w=None), km.ERR_NULL),
    (2, dict(cache_stride=(16 * 576, 572)), km.ERR_ALIGN),
    (2, dict(out=0x20000000), km.ERR_ALIAS),
    (2, dict(row_base=0x22000000), km.ERR_ALIAS),
    (2, dict(n_requests=1 << 24), km.ERR_RANGE),
    (3, {}, km.OK),
    (3, dict(n_requests=0, q=None), km.OK),
    (3, dict(n_queries=0, q=None), km.OK),
    (3, dict(latent_dim=384), km.ERR_UNSUPPORTED),
    (3, dict(rope_dim=32), km.ERR_UNSUPPORTED),
    (3, dict(n_heads=0), km.ERR_SHAPE),
    (3, dict(page_size=24), km.ERR_UNSUPPORTED),
    (3, dict(causal=2), km.ERR_SHAPE),
    (3, dict(window=-1), km.ERR_SHAPE),
    (3, dict(window=5, causal=0), km.ERR_SHAPE),
    (3, dict(scale=float("nan")), km.ERR_SHAPE),
    (3, dict(n_parts=1025), km.ERR_SHAPE),
    (3, dict(n_keys=2147483647, pt_stride=1 << 28), km.ERR_RANGE),
    (3, dict(pt_stride=255), km.ERR_SHAPE),
    (3, dict(page_table=None), km.ERR_NULL),
    (3, dict(cache=None), km.ERR_NULL),
    (3, dict(kv_tokens=None), km.ERR_NULL),
    (3, dict(q=0x20000002), km.ERR_ALIGN),
    (3, dict(cache_stride=(16 * 576, 580)), km.ERR_ALIGN),
    (3, dict(cache_stride=(16 * 576, -576)), km.ERR_RANGE),
    (3, dict(cache_stride=(16 * 576, 1 << 25)), km.ERR_RANGE),
    (3, dict(workspace=None), km.ERR_NULL),
    (3, dict(workspace_bytes=100), km.ERR_SHAPE),
    (3, dict(workspace=0x60000008), km.ERR_ALIGN),
    (3, dict(workspace=None, n_keys=64), km.OK),
    (3, dict(out=0x20000000), km.ERR_ALIAS),
    (3, dict(out=0x30000000), km.ERR_ALIAS),
    (3, dict(workspace=0x21000000), km.ERR_ALIAS),
    (3, dict(lse=0x21000000), km.ERR_ALIAS),
    (3, dict(q_tokens=0x21000000), km.ERR_ALIAS),
    (3, dict(n_requests=1 << 28), km.ERR_RANGE),
    (4, {}, km.OK),
    (4, dict(n_requests=0, k=None), km.OK),
    (4, dict(head_dim=96), km.ERR_UNSUPPORTED),
    (4, dict(rope_dim=128), km.ERR_UNSUPPORTED),
    (4, dict(k=None), km.ERR_NULL),
    (4, dict(rope_cache=None), km.ERR_NULL),
    (4, dict(v=0x48000008), km.ERR_ALIGN),
    (4, dict(k_stride=(1 << 25, 128)), km.ERR_RANGE),
    (4, dict(v_stride=(-2048, 128)), km.ERR_RANGE),
    (4, dict(out=0x40000000), km.ERR_ALIAS),
    (4, dict(out=0x48000000), km.ERR_ALIAS),
    (4, dict(kv_base=0x60000000), km.ERR_ALIAS),
    (4, dict(window=3, causal=0), km.ERR_SHAPE),
    # how many rows there are behind a base is not known: n_queries or n_keys rows may reach past the tensor
    (3, dict(q_base=P + 0x2000, n_queries=4096, out=0x20000000 + 2 * 2 * 16 * 576), km.OK),
    (3, dict(n_queries=4096, out=0x20000000 + 2 * 2 * 16 * 576), km.ERR_ALIAS),
    (4, dict(kv_base=P + 0x2000, workspace=0x40000000 + 2 * 2 * 16 * 128), km.OK),
    (4, dict(workspace=0x40000000 + 2 * 2 * 16 * 128), km.ERR_ALIAS),
]


@pytest.mark.parametrize("which,change,code", CASES)
def test_validation(which, change, code):
    a = MAKE[which](**change)
    assert km.lib().kamera_validate_latent(which, ctypes.byref(a)) == code, km.last_error()
    assert (km.last_error() == "") == (code == km.OK)


# Pools whose strides do not fall from the first dimension to the last, keys and values beside each other in every
# (page, layer), every token, every head: pages outermost, heads outermost, tokens outermost.
@pytest.mark.parametrize("order", ["page layer plane token head", "head page plane layer token", "token page layer plane head",
                                   "plane token head layer page", "page layer head token plane", "layer page token plane head"])
def test_keys_and_values_beside_each_other_in_any_order(order):
    size = dict(page=10, layer=3, token=16, head=4, plane=2)
    stride, at = {}, 128
    for d in reversed(order.split()):
        stride[d], at = at, at * size[d]
    strides = tuple(stride[d] for d in ("layer", "page", "token", "head"))

    def code(shift=0):
        a = rotate_args(k_cache_stride=strides, v_cache_stride=strides, v_cache=0x30000000 + 2 * (stride["plane"] + shift))
        return km.lib().kamera_validate_latent(0, ctypes.byref(a))

    assert code() == km.OK, km.last_error()
    for shift in (-8, 8, 64, -stride["plane"]):
        met = bool(_elements(0, strides, (3, 10, 16, 4), 128) & _elements(stride["plane"] + shift, strides, (3, 10, 16, 4), 128))
        assert not met or code(shift) == km.ERR_ALIAS, shift


def _elements(base, strides, sizes, width):
    x = [base]
    for s, n in zip(strides, sizes):
        x = [y + i * s for y in x for i in range(n)]
    return {y + c for y in x for c in range(0, width, 8)}


def test_bands_beside_each_other_in_packed_rows():
    """Queries' bands in and out in one tensor of rows behind row bases, of which no number is known."""
    def code(q_row, out_row, out_at, head=128):
        a = rotate_args(row_base=P + 0x100, k_stride=(0, 20480, 512, 128), v_stride=(0, 20480, 512, 128),
                        q_stride=(0, 1 << 20, q_row, head), q_out=0x22000000 + 2 * out_at, q_out_stride=(0, 1 << 20, out_row, head))
        return km.lib().kamera_validate_latent(0, ctypes.byref(a))

    assert code(1024, 1024, 64) == km.OK, km.last_error()        # columns of a head
    assert code(2048, 2048, 1024) == km.OK, km.last_error()      # heads of a row
    assert code(1024, 1024, 1 << 19) == km.OK, km.last_error()   # rows of a layer
    assert code(1024, 2048, 64) == km.OK, km.last_error()        # every other row's
    assert code(1024, 1024, 56) == km.ERR_ALIAS
    assert code(1000, 1024, 64) == km.ERR_ALIAS                  # the second rows meet


def test_outputs_that_meet_are_refused_whatever_their_strides():
    """Two pools at random strides, also 0 and negative ones, and distances: every pair that shares memory is refused."""
    rng = random.Random(0)
    sizes, allowed = (2, 3, 4, 2), 0
    for _ in range(3000):
        dims = [0, 1, 2, 3, 4]
        rng.shuffle(dims)                          # 4: keys or values
        stride, at = [0] * 5, 16
        for d in dims:
            stride[d] = at * rng.choice((1, 1, 1, 1, 1, -1))
            at *= (2 if d == 4 else sizes[d]) + rng.choice((0, 0, 0, 1))
        other = list(stride)
        if rng.random() < 0.3:
            other[rng.randrange(4)] = 8 * rng.randrange(-6, 12)
        apart = stride[4] + 8 * rng.choice((0, 0, 0, 1, -1, 3, rng.randrange(-40, 40)))
        a = rotate_args(n_layers=2, n_pool_pages=3, page_size=4, n_k_heads=2, n_v_heads=2, k_dim=16, v_dim=16, pt_stride=16,
                        k_cache_stride=tuple(stride[:4]), v_cache_stride=tuple(other[:4]), v_cache=0x30000000 + 2 * apart, q=None,
                        q_out=None, **{"rope.rope_dim": 16})
        code = km.lib().kamera_validate_latent(0, ctypes.byref(a))
        assert code in (km.OK, km.ERR_ALIAS), km.last_error()
        if code == km.OK:
            allowed += 1
            assert not _elements(0, stride, sizes, 16) & _elements(apart, other, sizes, 16), (stride, other, apart)
    assert allowed > 500


def test_launches_past_32_bits_of_threads_are_refused():
    """A workgroup of the latent form has 256 threads, 512 where a block has more than 32 rows; of the expanded 256."""
    def code(which, requests, **kw):
        a = MAKE[which](n_requests=requests, n_keys=16, pt_stride=1, workspace=None, q_base=P, **kw)
        return km.lib().kamera_validate_latent(which, ctypes.byref(a))

    for heads, block, threads in ((16, 16, 256), (32, 32, 256), (48, 128, 512), (128, 128, 512)):
        for n_queries in (1, 1 << 17) if heads == 128 else (1,):
            blocks = -(-n_queries * heads // block)              # of a request; a workgroup each
            most = (1 << 32) // threads // blocks
            assert code(3, most, n_heads=heads, n_queries=n_queries) == km.ERR_RANGE
            assert code(3, most - 16, n_heads=heads, n_queries=n_queries) == km.OK, km.last_error()
    assert code(4, 1 << 20, kv_base=P) == km.ERR_RANGE           # 2^20 requests of 16 heads
    assert code(4, (1 << 20) - 1, kv_base=P) == km.OK, km.last_error()


def test_validation_of_nothing():
    L = km.lib()
    for which in range(5):
        assert L.kamera_validate_latent(which, None) == km.ERR_NULL
    assert L.kamera_validate_latent(5, None) == km.ERR_SHAPE
    assert L.kamera_attend_latent_workspace(None) == km.ERR_NULL
    assert L.kamera_attend_expanded_workspace(None) == km.ERR_NULL


def test_struct_layout():
    for which, cls in latent.STRUCTS.items():
        assert km.lib().kamera_struct_size(which) == ctypes.sizeof(cls)


def test_workspace():
    L = km.lib()
    a = latent_args(n_parts=5)
    # two segments of a workgroup, a block's rows (16 of each wave): sums, and four words; then the
    # tasks' and the workgroups' places
    assert L.kamera_attend_latent_workspace(ctypes.byref(a)) == 5 * 2 * 16 * (512 + 4) * 4 + 32
    a = latent_args(n_parts=3, n_queries=9)                      # 144 rows: two blocks of 128 for each request
    assert L.kamera_attend_latent_workspace(ctypes.byref(a)) == 3 * 2 * 128 * (512 + 4) * 4 + 32
    a = expanded_args(n_parts=4)
    assert L.kamera_attend_expanded_workspace(ctypes.byref(a)) == 4 * 2 * 128 * (128 + 4) * 4 + 160
    # short contexts, and enough work for all: a workgroup takes a block's keys whole
    assert L.kamera_attend_latent_workspace(ctypes.byref(latent_args(n_keys=64))) == 0
    assert L.kamera_attend_latent_workspace(ctypes.byref(latent_args(n_requests=4000))) == 0
    assert L.kamera_attend_expanded_workspace(ctypes.byref(expanded_args(n_requests=1000))) == 0
    assert L.kamera_attend_latent_workspace(ctypes.byref(latent_args(latent_dim=500))) == km.ERR_UNSUPPORTED


def test_scaled_frequencies_against_their_definition():
    """The tests' own frequencies at the definitions' borders."""
    f = ref.frequencies(1e4, 64)
    turns = 4096 * f / (2 * math.pi)
    g = ref.frequencies(1e4, 64, "turns", 4.0, 4096, 1.0, 4.0)
    assert (g[turns >= 4] == f[turns >= 4]).all()
    assert abs(g[turns <= 1] / f[turns <= 1] - 0.25).max() < 1e-15
    h = ref.frequencies(1e4, 64, "pairs", 40.0, 4096, 1.0, 32.0)
    assert h[0] == f[0] and abs(h[-1] * 40 / f[-1] - 1) < 1e-15
    assert (abs(h[1:]) < abs(h[:-1])).all()


def test_binding_refuses():
    """Types, shapes and layouts that the binding itself turns down, on CPU tensors."""
    bf, i4 = torch.bfloat16, torch.int32
    table, kv = torch.zeros((2, 3), dtype=i4), torch.zeros(2, dtype=i4)
    rope = km.RopeSpec(theta=1e4, rope_dim=64)
    k = torch.zeros((2, 1, 5, 2, 64), dtype=bf)
    pool = torch.zeros((1, 4, 16, 2, 64), dtype=bf)

    def append(**kw):
        a = dict(k=k, v=k.clone(), k_cache=pool, v_cache=pool.clone(), page_table=table, rope=rope)
        a.update(kw)
        km.prepare_append_rotated(a.pop("k"), a.pop("v"), a.pop("k_cache"), a.pop("v_cache"), a.pop("page_table"), **a)

    with pytest.raises(ValueError, match="device memory"):
        append()
    for bad, err in ((dict(k=k.float()), TypeError), (dict(k=k[0]), ValueError), (dict(v=k[:, :, :3]), ValueError),
                     (dict(k_cache=pool[..., :32]), ValueError), (dict(v_cache=pool[:, :2]), ValueError),
                     (dict(v_cache=None), ValueError), (dict(q=k), ValueError), (dict(q=k[..., :32], q_out=k[..., :32]), ValueError),
                     (dict(page_table=table.long()), TypeError), (dict(n_tokens=6), ValueError), (dict(n_tokens=1 << 32), ValueError),
                     (dict(tokens_before=kv.long()), TypeError), (dict(row_base=kv), ValueError),
                     (dict(positions=torch.zeros((2, 4), dtype=i4)), ValueError),
                     (dict(positions=torch.zeros((2, 5))), TypeError),
                     (dict(positions=torch.zeros((2, 5, 3), dtype=i4)), ValueError),
                     (dict(scaling=km.RopeScaling("linear", 2.0, amplitude=0.0)), ValueError),
                     (dict(scaling=km.RopeScaling("cubic", 2.0)), KeyError)):
        with pytest.raises(err):
            append(**bad)

    x, w, out = torch.zeros((3, 2, 64), dtype=bf), torch.zeros((2, 64, 128), dtype=bf), torch.zeros((3, 2, 128), dtype=bf)
    for bad in ((x.float(), w, out), (x, w.float(), out), (x, w[:1], out), (x, w[:, :32], out), (x, w, out[..., :64]),
                (x[0], w, out), (x, w, out[:2])):
        with pytest.raises((TypeError, ValueError)):
            km.prepare_project_heads(*bad)
    with pytest.raises(ValueError, match="device memory"):
        km.prepare_project_heads(x, w, out)

    rows = torch.zeros((4, 16, 320), dtype=bf)
    for bad in (dict(cache=rows[..., :32]), dict(out=out[..., :64]), dict(n_keys=40), dict(kv=kv.long()), dict(cache=rows.float()),
                dict(cache=rows[0])):
        a = dict(cache=rows, w=w, out=torch.zeros((70, 2, 128), dtype=bf), kv=kv, n_keys=35)
        a.update(bad)
        with pytest.raises((TypeError, ValueError)):
            km.prepare_expand_latent(a["cache"], a["w"], a["out"], table, a["kv"], n_keys=a["n_keys"])

    q, o = torch.zeros((2, 4, 320), dtype=bf), torch.zeros((2, 4, 256), dtype=bf)

    def attend(**kw):
        a = dict(q=q, cache=rows, out=o, n_queries=1, n_keys=40, scale=0.1)
        a.update(kw)
        km.prepare_attend_latent(a.pop("q"), a.pop("cache"), a.pop("out"), table, a.pop("kv", kv), **a)

    with pytest.raises(ValueError, match="device memory"):
        attend()
    for bad, err in ((dict(q=q.float()), TypeError), (dict(out=o[:1]), ValueError), (dict(cache=rows[..., :300]), ValueError),
                     (dict(out=o[..., :192]), km.KameraError), (dict(kv=kv.long()), TypeError), (dict(n_queries=2), ValueError),
                     (dict(lse=torch.zeros(2, 4, dtype=bf)), TypeError), (dict(lse=torch.zeros(4, 2)), ValueError),
                     (dict(window=-2), km.KameraError), (dict(n_keys=-1), km.KameraError), (dict(n_keys=1 << 32), ValueError),
                     (dict(n_parts=1 << 32), ValueError), (dict(q_base=kv.long()), TypeError),
                     (dict(workspace=torch.zeros(8)[::2]), ValueError)):
        with pytest.raises(err):
            attend(**bad)

    qe, oe, e = torch.zeros((2, 4, 128), dtype=bf), torch.zeros((2, 4, 64), dtype=bf), torch.zeros((80, 4, 128), dtype=bf)

    def expanded(**kw):
        a = dict(q=qe, k=e[..., :64], v=e[..., 64:], rope=rows[..., -64:], out=oe, n_queries=1, n_keys=40, scale=0.1)
        a.update(kw)
        km.prepare_attend_expanded(a.pop("q"), a.pop("k"), a.pop("v"), a.pop("rope"), a.pop("out"), table, kv, **a)

    with pytest.raises(ValueError, match="device memory"):
        expanded()
    for bad in (dict(k=e), dict(v=e[:3, :, :64]), dict(rope=rows), dict(out=oe[:, :2]), dict(n_keys=41), dict(kv_base=kv.long()),
                dict(q=qe[0]), dict(k=e[:, :2, :64], v=e[:, :2, 64:])):
        with pytest.raises((TypeError, ValueError)):
            expanded(**bad)


def test_views_of_page_tables_end_where_the_view_does(monkeypatch):
    monkeypatch.setattr(latent, "_device", lambda *t: None)
    whole = torch.zeros((2, 20), dtype=torch.int32)
    k = torch.zeros((2, 1, 5, 1, 64), dtype=torch.bfloat16)
    pool = torch.zeros((1, 4, 16, 1, 64), dtype=torch.bfloat16)
    q, o = torch.zeros((2, 4, 320), dtype=torch.bfloat16), torch.zeros((2, 4, 256), dtype=torch.bfloat16)
    rows, kv = torch.zeros((4, 16, 320), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    for view in (whole[:, :2], whole[:, 18:], whole):
        a = km.prepare_append_rotated(k, None, pool, None, view, rope=km.RopeSpec(theta=1e4, rope_dim=64)).args
        assert (a.pt_stride, a.pt_pages) == (20, view.shape[1])
        a = km.prepare_attend_latent(q, rows, o, view, kv, n_queries=1, n_keys=32, scale=0.1).args
        assert a.pt_stride == 20
    with pytest.raises(ValueError, match="hold less"):
        km.prepare_attend_latent(q, rows, o, whole[:, :2], kv, n_queries=1, n_keys=33, scale=0.1)


def _host_program(tmp_path, name, flags):
    if shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("no g++ or HIP headers")
    exe = str(tmp_path / name)
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-D__HIP_PLATFORM_AMD__", "-I",
           "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", TC, *flags,
           *[os.path.join(CSRC, f) for f in ("kamera_abi.cpp", "kamera_latent.cpp")],
           *[os.path.join(TC, f) for f in ("launch_stub.cpp", "latent_stub.cpp", "latent_sanitize.cpp")], "-o", exe, "-pthread"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300,
                       env=dict(os.environ, UBSAN_OPTIONS="print_stacktrace=1", TSAN_OPTIONS="halt_on_error=1"))
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), (r.stdout[-2000:], r.stderr[-4000:])


def test_host_layer_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    _host_program(tmp_path, "latent_asan", ["-fsanitize=address,undefined", "-fno-sanitize-recover=undefined"])


def test_host_layer_under_thread_sanitizer(tmp_path):
    _host_program(tmp_path, "latent_tsan", ["-fsanitize=thread"])


MIXED_LOADS = """
#include "kamera_lds_device.h"
using namespace kamera;
// a load into LDS by the compiler, one by load_lds, and one by the compiler to the first one's place
template <bool PAIR>
__global__ void mixed_loads(const uint8_t* a, const uint8_t* b, uint32_t* out) {
  __shared__ uint32_t s[4096];
  const auto lds = (__attribute__((address_space(3))) void*)s;
  __builtin_amdgcn_global_load_lds((GlobalBytes)(a + threadIdx.x * 16), lds, 16, 0, 0);
  if (PAIR) load_lds(b, threadIdx.x * 16, lds_offset(s) + 4096);
  else load_lds((uint64_t)b + threadIdx.x * 16, lds_offset(s) + 4096);
  __builtin_amdgcn_global_load_lds((GlobalBytes)(a + 4096 + threadIdx.x * 16), lds, 16, 64, 0);
  vm_wait<0>();
  out[threadIdx.x] = s[threadIdx.x + 64];
}
template __global__ void mixed_loads<true>(const uint8_t*, const uint8_t*, uint32_t*);
template __global__ void mixed_loads<false>(const uint8_t*, const uint8_t*, uint32_t*);
"""


def test_loads_into_lds_say_that_they_write_m0(tmp_path):
    """load_lds sets m0, which holds the place in LDS of every such load: the compiler, which sets it for its own ones,
    has to set it anew behind it."""
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    src, asm = tmp_path / "mixed_loads.hip", tmp_path / "mixed_loads.s"
    src.write_text(MIXED_LOADS)
    r = subprocess.run([hipcc, "-S", "--cuda-device-only", "-O3", "--offload-arch=gfx950", "-std=c++17", "-I",
                        os.path.join(ROOT, "include"), "-I", CSRC, str(src), "-o", str(asm)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    kernels = [k.split("s_endpgm")[0] for k in asm.read_text().split("; -- Begin function")[1:]]
    assert len(kernels) == 2
    for k in kernels:
        loads = k.split("global_load_lds_dwordx4")
        assert len(loads) == 4                                   # three loads, m0 set before each
        assert all("s_mov_b32 m0" in before for before in loads[:3]), k


def test_tiles_of_the_products(tmp_path):
    """The tile that the host picks for the shapes of the GPU tests of each one."""
    from tests import test_gpu_latent as gpu

    if shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("no g++ or HIP headers")
    exe = str(tmp_path / "latent_params")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I",
                        os.path.join(ROOT, "include"), "-I", CSRC, "-I", TC,
                        *[os.path.join(CSRC, f) for f in ("kamera_abi.cpp", "kamera_latent.cpp")],
                        *[os.path.join(TC, f) for f in ("launch_stub.cpp", "latent_params.cpp")], "-o", exe, "-pthread"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    calls = [("project", 1, *c, 256) for c in gpu.PROJECT_256]
    calls += [("expand", len(c[0]), max(c[0]), *c[2:], 256) for c in gpu.EXPAND_256]
    calls += [("project", 1, 64, 16, 128, 512, 32), ("project", 1, 65, 3, 64, 192, 128), ("expand", 4, 300, 4, 256, 256, 128)]
    for *call, rows in calls:
        r = subprocess.run([exe, *map(str, call)], capture_output=True, text=True, timeout=60)
        assert r.returncode == 0 and int(r.stdout) == rows, (call, r.stdout, r.stderr)
