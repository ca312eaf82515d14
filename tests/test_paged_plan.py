"""Checks of the paged calls' arguments (csrc/paged_plan.h), compiled by the host compiler and asked without a GPU,
and those of the Python binding."""
import ctypes as C
import math
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2510_10129_amd as cc
from oracle import paged
from paper_2510_10129_amd import _lib, build
from paper_2510_10129_amd._lib import (CC_ERR_NULL, CC_ERR_SHAPE, CC_ERR_WORKSPACE, CC_OK, _NewRows, _PagedKV, _Pool, _Rope)

CXX = shutil.which("g++") or shutil.which("c++")

SHIM = r"""
#include "paged_plan.h"
extern "C" {
int pool(const cc_page_pool* p) { return cc_check_pool(p).code; }
int layers(const cc_paged_kv* kv, int n, int page, int H_kv, int d_h) { return cc_check_layers(kv, n, page, H_kv, d_h).code; }
int list(int n, int n_seqs, const int32_t* a, const int32_t* b) { return cc_check_list(n, n_seqs, a, b).code; }
int new_rows(const cc_new_rows* r, int n_seqs, int g) { return cc_check_new_rows(r, n_seqs, g).code; }
int rope(const cc_rope* r, int d_h) { return cc_check_rope(r, d_h).code; }
void turns(const cc_rope* r, double* out) { cc_rope_turns(*r, out); }
int overlap(const void* a, int64_t na, const void* b, int64_t nb) { return cc_overlap(a, na, b, nb); }
int64_t work(int n_pages, int n_seqs) { return cc_page_work_size(n_pages, n_seqs); }
void layout(int n_pages, int n_seqs, int64_t* o) {
    const cc_page_work w = cc_page_work_layout(n_pages, n_seqs);
    const int64_t v[] = {w.take, w.first, w.copy_at, w.list, w.map, w.src, w.dst, w.rows, w.attn, w.ints};
    for (int i = 0; i < 10; ++i) o[i] = v[i];
}
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if CXX is None:
        pytest.skip("no host C++ compiler")
    d = tmp_path_factory.mktemp("paged")
    (d / "shim.cpp").write_text(SHIM)
    cmd = [CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", build.CSRC, "-I", build.ROOT + "/include",
           str(d / "shim.cpp"), "-o", str(d / "shim.so")]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    so = C.CDLL(str(d / "shim.so"))
    so.work.restype = C.c_int64
    return so


A = 1 << 20            # an aligned address that nothing reads


def _pool(**kw):
    f = dict(refs=A, table=A, len=A, status=A, work=A, work_bytes=1 << 40, stride_table=8, n_pages=64, page_size=16, n_seqs=4,
             max_pages=8)
    f.update(kw)
    return _Pool(**f)


def test_pool_checks(lib):
    assert lib.pool(C.byref(_pool())) == CC_OK and lib.pool(None) == CC_ERR_NULL
    for name in ("refs", "table", "len", "status", "work"):
        assert lib.pool(C.byref(_pool(**{name: None}))) == CC_ERR_NULL
    for bad in (dict(page_size=8), dict(page_size=24), dict(page_size=2048), dict(n_pages=0), dict(n_seqs=0), dict(n_seqs=65537),
                dict(max_pages=0), dict(stride_table=7), dict(work=A + 64), dict(table=A + 2), dict(n_pages=1 << 27),
                dict(max_pages=1 << 26, stride_table=1 << 26), dict(n_pages=-1), dict(page_size=-16)):
        assert lib.pool(C.byref(_pool(**bad))) == CC_ERR_SHAPE, bad
    need = lib.work(64, 4)
    assert need == _lib.load_library().cc_page_work_bytes(64, 4) > 0
    assert lib.pool(C.byref(_pool(work_bytes=need - 1))) == CC_ERR_WORKSPACE and lib.pool(C.byref(_pool(work_bytes=need))) == CC_OK
    assert lib.pool(C.byref(_pool(page_size=1024, n_pages=(1 << 21) - 1, max_pages=(1 << 20) - 1, stride_table=1 << 20))) == CC_OK
    assert _lib.load_library().cc_page_work_bytes(0, 4) == 0


@pytest.mark.parametrize("n_pages,n_seqs", [(1, 1), (64, 4), (7, 300), (100000, 65536)])
def test_scratch_regions_do_not_overlap(lib, n_pages, n_seqs):
    o = (C.c_int64 * 10)()
    lib.layout(n_pages, n_seqs, o)
    sizes = [n_seqs] * 3 + [n_pages] * 2 + [max(n_pages, n_seqs)] * 3
    assert o[0] >= 2
    for i, n in enumerate(sizes):
        assert o[i] + n <= o[i + 1], i
    assert o[8] <= o[9] and lib.work(n_pages, n_seqs) == 4 * o[9]


def test_layer_checks(lib):
    def kv(**kw):
        f = dict(K=A, V=A, stride_page=16 * 4 * 128, stride_token=4 * 128, stride_head=128)
        f.update(kw)
        return _PagedKV(**f)

    def code(*kvs):
        return lib.layers((_PagedKV * len(kvs))(*kvs), len(kvs), 16, 4, 128)

    assert code(kv()) == code(kv(), kv()) == code() == CC_OK
    assert code(kv(stride_token=128, stride_head=16 * 128)) == CC_OK                     # heads outermost
    assert code(kv(stride_page=1 << 33)) == CC_OK
    assert code(kv(K=None)) == CC_ERR_NULL and lib.layers(None, 1, 16, 4, 128) == CC_ERR_NULL
    for bad in (dict(stride_page=16 * 4 * 128 - 8), dict(stride_token=4 * 128 + 4), dict(stride_head=120), dict(stride_token=64),
                dict(stride_head=256), dict(K=A + 8), dict(V=A + 2), dict(stride_page=0), dict(stride_page=-8),
                dict(stride_token=1 << 23, stride_page=1 << 28)):
        assert code(kv(**bad)) == CC_ERR_SHAPE, bad
    assert code(kv(), kv(stride_page=1 << 20)) == CC_ERR_SHAPE and lib.layers(None, -1, 16, 4, 128) == CC_ERR_SHAPE


def test_list_and_row_checks(lib):
    a = C.cast(A, C.POINTER(C.c_int32))
    assert lib.list(4, 4, a, a) == CC_OK and lib.list(0, 4, None, None) == CC_OK
    assert lib.list(5, 4, a, a) == lib.list(-1, 4, a, a) == CC_ERR_SHAPE and lib.list(1, 4, a, None) == CC_ERR_NULL

    def rows(g=4, n_seqs=4096, **kw):
        f = dict(start=A, seq=A, n=3, rows=10, max_new=4)
        f.update(kw)
        return lib.new_rows(C.byref(_NewRows(**f)), n_seqs, g)

    assert rows() == rows(seq=None) == rows(n=0, start=None) == rows(n=1024) == rows(rows=0) == rows(rows=1 << 18) == CC_OK
    assert lib.new_rows(None, 4, 1) == rows(start=None) == CC_ERR_NULL
    for bad in (dict(n=-1), dict(n=1025), dict(rows=-1), dict(max_new=-1), dict(rows=(1 << 18) + 1), dict(seq=None, n_seqs=2),
                dict(start=A + 2), dict(seq=A + 1)):
        assert rows(**bad) == CC_ERR_SHAPE, bad


def test_rope_checks(lib):
    good = dict(base=1e4, rot=64, interleaved=0, scaling=3, orig_len=8192, factor=8.0, low=1.0, high=32.0, mscale=1.2)
    assert lib.rope(C.byref(_Rope(**good)), 64) == CC_OK and lib.rope(None, 64) == CC_ERR_NULL
    for bad in (dict(base=1.0), dict(base=math.nan), dict(base=math.inf), dict(rot=0), dict(rot=66), dict(rot=7), dict(scaling=4),
                dict(scaling=-1), dict(factor=0.5), dict(factor=math.nan), dict(orig_len=0), dict(low=0.0), dict(high=1.0),
                dict(high=math.inf), dict(mscale=math.nan)):
        assert lib.rope(C.byref(_Rope(**{**good, **bad})), 64) == CC_ERR_SHAPE, bad
    assert lib.rope(C.byref(_Rope(base=1e4, rot=2, mscale=1.0)), 64) == CC_OK               # plain: the rest is not looked at


@pytest.mark.parametrize("kind", _lib.ROPE_SCALINGS)
@pytest.mark.parametrize("base,rot,orig,low,high", [(1e4, 64, 8192, 1.0, 32.0), (5e5, 128, 4096, 1.0, 4.0), (1e6, 2, 100, 0.5, 3.0),
                                                    (1.5, 30, 1, 1.0, 1.001)])
def test_rope_frequencies(lib, kind, base, rot, orig, low, high):
    rule = cc.Rope(base, rot, False, kind, 8.0, orig, low, high)
    out = (C.c_double * 64)()
    lib.turns(C.byref(rule.c_struct()), out)
    ref = paged.frequencies(base, rot, kind, 8.0, orig, low, high) / (2 * math.pi)
    assert np.allclose(out[:rot // 2], ref, rtol=1e-12)


def test_overlap(lib):
    def over(a, n_a, b, n_b):
        assert lib.overlap(C.c_void_p(a), C.c_int64(n_a), C.c_void_p(b), C.c_int64(n_b)) == lib.overlap(
            C.c_void_p(b), C.c_int64(n_b), C.c_void_p(a), C.c_int64(n_a))
        return lib.overlap(C.c_void_p(a), C.c_int64(n_a), C.c_void_p(b), C.c_int64(n_b))

    assert over(A, 8, A, 8) and over(A, 9, A + 16, 8) and over(A, 100, A + 32, 1) and over(A, 1 << 32, A + (1 << 33) - 2, 1)
    assert not over(A, 8, A + 16, 8) and not over(A, 0, A, 8) and not over(A, 1 << 32, A + (1 << 33), 1)


def _torch_pool(n_pages=8, page=16, n_seqs=3, max_pages=4):
    return cc.PagePool.empty(n_pages, page, n_seqs, max_pages, device="cpu")


def test_binding_refuses_what_the_library_cannot_read():
    P = _torch_pool()
    assert P.work.numel() == _lib.load_library().cc_page_work_bytes(8, 3)
    i32 = dict(dtype=torch.int32)
    with pytest.raises(ValueError):
        cc.PagePool(P.refs.long(), P.table, P.len, 16)
    with pytest.raises(ValueError):
        cc.PagePool(P.refs, P.table[:2], P.len, 16)
    with pytest.raises(ValueError):
        cc.PagePool(P.refs, torch.zeros(4, 3, **i32).t(), P.len, 16)
    with pytest.raises(ValueError):
        cc.PagePool(torch.zeros(16, **i32)[::2], P.table, P.len, 16)
    m = _lib.ModelDesc(64, 4, 2, 64, 64, 1e4, 1e-5, 64, 64, 64)
    K = torch.zeros(8, 16, 2, 64, dtype=torch.bfloat16)
    assert cc.PagedKV.table([cc.PagedKV(K, K)], P, m).tolist()[2:] == [16 * 2 * 64, 2 * 64, 64]
    by_head = torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16).transpose(1, 2)
    assert cc.PagedKV.table([cc.PagedKV(by_head, by_head)], P, m).tolist()[2:] == [16 * 2 * 64, 64, 16 * 64]
    for bad in (K.float(), K[:4], K[..., :32], K.transpose(2, 3).contiguous().transpose(2, 3), by_head):
        with pytest.raises(ValueError):
            cc.PagedKV.table([cc.PagedKV(K, bad)], P, m)
    for other in (_torch_pool(n_pages=9), _torch_pool(page=32)):
        with pytest.raises(ValueError):
            cc.PagedKV.table([cc.PagedKV(K, K)], other, m)
    kv = cc.PagedKV(K, K)
    cc.PagedKV.table([kv], P, m)
    kv.K = kv.V = by_head                                   # an assigned field is looked at again
    assert cc.PagedKV.table([kv], P, m)[4] == 16 * 64
    start = torch.zeros(3, **i32)
    assert cc.NewRows(start, None, 4, 2).c_struct().n == 2
    for s, q in ((start, torch.zeros(3, **i32)), (start.float(), None), (start[:0], None), (torch.zeros(6, **i32)[::2], None)):
        with pytest.raises(ValueError):
            cc.NewRows(s, q, 4, 2).c_struct()
    with pytest.raises(ValueError):
        cc.Rope(1e4, 64, scaling="other").c_struct()


class _NoCalls:
    def __getattr__(self, name):
        raise AssertionError("the library was called")


def test_binding_checks_buffers_before_the_call():
    P, bf = _torch_pool(), dict(dtype=torch.bfloat16)
    ctx = _lib.Context.__new__(_lib.Context)
    ctx._lib, ctx._h = _NoCalls(), None
    ctx.desc = _lib.ModelDesc(64, 4, 2, 64, 64, 1e4, 1e-5, 64, 64, 64)
    K = torch.zeros(8, 16, 2, 64, **bf)
    kv, new = cc.PagedKV(K, K), cc.NewRows(torch.zeros(2, dtype=torch.int32), None, 5, 5)
    q, k, rule = torch.zeros(5, 256, **bf), torch.zeros(5, 128, **bf), cc.Rope(1e4, 64)
    for bad in (q.float(), q[:4], q[:, :128], torch.zeros(256, 5, **bf).t(), torch.zeros(5, 512, **bf)[:, :256]):
        with pytest.raises(ValueError):
            ctx.step_paged_attention(bad, new, P, kv, q)
        with pytest.raises(ValueError):
            ctx.step_paged_attention(q, new, P, kv, bad)
    for args in ((q[:4], k, k, q), (q, k[:, :64], k, q), (q, k, k.float(), q), (q, k, k, torch.zeros(5, 512, **bf)[:, :256])):
        with pytest.raises(ValueError):
            ctx.step_rope_append(*args[:3], new, P, kv, rule, args[3])
    with pytest.raises(ValueError):
        ctx.step_rope_append(q, k, k, new, P, kv, rule, q, pos=torch.zeros(4, dtype=torch.int32))
    one = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        ctx._seqs(P, one, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        ctx._seqs(P, one.long(), one)


def test_null_context_is_refused():
    so = _lib.load_library()
    assert so.cc_grow_pages(None, None, None, 0, None, None, 0, None) == CC_ERR_NULL
    assert so.cc_fork_pages(None, None, None, None, 0, None) == CC_ERR_NULL
    assert so.cc_free_pages(None, None, None, 0, None) == CC_ERR_NULL
    assert so.cc_compact_pages(None, None, None, 0, None) == CC_ERR_NULL
    assert so.cc_step_rope_append(None, None, 0, None, 0, None, 0, None, None, None, None, None, None, 0) == CC_ERR_NULL
    assert so.cc_step_paged_attention(None, None, None, None, None, 0, 0, None, 0) == CC_ERR_NULL
