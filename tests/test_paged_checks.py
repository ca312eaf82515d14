"""More checks of the paged calls' arguments (csrc/paged_plan.h), compiled by the host compiler and asked without a GPU."""
import ctypes as C
import subprocess

import pytest
import torch

import paper_2510_10129_amd as cc
from paper_2510_10129_amd import _lib, build
from paper_2510_10129_amd._lib import CC_ERR_NULL, CC_ERR_SHAPE, CC_OK, _NewRows, _Pool, _Rope

from test_paged_plan import A, CXX, _pool

SHIM = r"""
#include "paged_plan.h"
extern "C" {
int pool(const cc_page_pool* p) { return cc_check_pool(p).code; }
int grow(const cc_page_pool* p, const int32_t* status) { return cc_check_grow(*p, status).code; }
int rope(const cc_rope* r, int d_h) { return cc_check_rope(r, d_h).code; }
int pool_size() { return sizeof(cc_page_pool); }
int attend(const cc_new_rows* r, const cc_page_pool* p, int g, int window, int sinks) { return cc_check_attend(*r, *p, g, window, sinks).code; }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if CXX is None:
        pytest.skip("no host C++ compiler")
    d = tmp_path_factory.mktemp("paged_checks")
    (d / "shim.cpp").write_text(SHIM)
    cmd = [CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", build.CSRC, "-I", build.ROOT + "/include",
           str(d / "shim.cpp"), "-o", str(d / "shim.so")]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    return C.CDLL(str(d / "shim.so"))


def test_a_grow_that_is_not_waited_for_says_what_it_refused(lib):
    assert lib.pool_size() == C.sizeof(_Pool)
    status = C.byref(C.c_int32())
    assert lib.grow(C.byref(_pool()), status) == lib.grow(C.byref(_pool(refused=A)), status) == CC_OK
    assert lib.grow(C.byref(_pool(refused=A)), None) == CC_OK and lib.grow(C.byref(_pool()), None) == CC_ERR_NULL
    assert lib.pool(C.byref(_pool(refused=A))) == CC_OK and lib.pool(C.byref(_pool(refused=A + 2))) == CC_ERR_SHAPE


def test_a_scale_that_32_bits_cannot_hold(lib):
    for mscale, code in ((3e38, CC_OK), (-3e38, CC_OK), (1e39, CC_ERR_SHAPE), (-1e300, CC_ERR_SHAPE), (float("inf"), CC_ERR_SHAPE),
                         (float("nan"), CC_ERR_SHAPE)):
        assert lib.rope(C.byref(_Rope(base=1e4, rot=2, mscale=mscale)), 64) == code, mscale


def _attend(lib, rows, n, max_pages, page=64, g=1, window=0, sinks=0):
    return lib.attend(C.byref(_NewRows(A, A, n, rows, 1)), C.byref(_pool(max_pages=max_pages, page_size=page, stride_table=1 << 26)), g, window, sinks)


def test_attention_checks(lib):
    assert _attend(lib, 10, 3, 8) == _attend(lib, 10, 3, 8, window=2 ** 31 - 1, sinks=2 ** 31 - 1) == _attend(lib, 0, 0, 8) == CC_OK
    assert _attend(lib, 10, 3, 8, window=-1) == _attend(lib, 10, 3, 8, sinks=-1) == CC_ERR_SHAPE
    # blocks times tiles below 2^31: 128 sequences of a row, 2^24 tiles of 64 keys with the 8 that a block costs besides its own
    for rows, n, g in ((128, 128, 1), (127 * 256, 1, 1), (127 * 32, 1, 8), (64 * 32, 64, 8)):
        assert _attend(lib, rows, n, (1 << 24) - 9, g=g) == CC_OK
        assert _attend(lib, rows, n, (1 << 24) - 8, g=g) == CC_ERR_SHAPE
    # 64 keys a tile, whatever the page
    assert _attend(lib, 128, 128, 4 * ((1 << 24) - 9), page=16) == CC_OK and _attend(lib, 128, 128, 4 * ((1 << 24) - 9) + 1, page=16) == CC_ERR_SHAPE


def test_units_of_the_largest_attention_call_fit_32_bits(lib):
    """The many-rows kernel counts key tiles in 32 bits: its blocks' tiles, 5 more a block, rounded up to whole ranges where no more
    blocks than workgroups are there (ranges of the longest block over the workgroups that a block can have, 8 at least)."""
    for n in list(range(1, 300)) + [511, 512, 1000, 1024]:
        tiles = min((1 << 24) - 1, (2 ** 31 - 1) // n - 8)
        assert _attend(lib, 0, n, tiles) == CC_OK and (tiles == (1 << 24) - 1 or _attend(lib, 0, n, tiles + 1) == CC_ERR_SHAPE)
        length = tiles + 5
        for workgroups in (64, 128, 256):
            for heads in (1, 2, 4, 8):
                units = n * length
                if n * heads <= workgroups:
                    each = max(8, -(-length // (workgroups // (n * heads))))
                    units = n * (-(-length // each) * each)
                assert units < 2 ** 31, (n, workgroups, heads)


def test_assigned_fields_of_a_pool_are_checked():
    """A pool whose tables were replaced is looked at again before the library is told of it."""
    i32 = dict(dtype=torch.int32)

    def assigned(**fields):
        p = cc.PagePool.empty(8, 16, 3, 4, device="cpu")
        p.c_struct()
        for name, t in fields.items():
            setattr(p, name, t)
        return p.c_struct()

    for bad in (dict(refs=torch.zeros(8, dtype=torch.int64)), dict(refs=torch.zeros(16, **i32)[::2]), dict(refs=torch.zeros(2, 4, **i32)),
                dict(table=torch.zeros(3, 4, dtype=torch.int64)), dict(table=torch.zeros(2, 4, **i32)), dict(table=torch.zeros(4, 3, **i32).t()),
                dict(table=torch.zeros(12, **i32)), dict(len=torch.zeros(3, dtype=torch.float64)), dict(len=torch.zeros(99, **i32)),
                dict(table=torch.zeros(2, 4, dtype=torch.int64), len=torch.zeros(99, dtype=torch.float64)),
                dict(table=torch.zeros(5, 4, **i32), len=torch.zeros(5, **i32)), dict(status=torch.zeros(1)), dict(status=torch.zeros(0, **i32)),
                dict(work=torch.zeros(64, 64, dtype=torch.uint8).t()), dict(refused=torch.zeros(3)), dict(refused=torch.zeros(2, **i32))):
        with pytest.raises(ValueError):
            assigned(**bad)
    longer = assigned(table=torch.zeros(5, 6, **i32), len=torch.zeros(5, **i32), refused=torch.zeros(5, **i32))
    assert (longer.n_seqs, longer.max_pages, longer.stride_table) == (5, 6, 6)


class _NoCalls:
    def __getattr__(self, name):
        return lambda *args: pytest.fail("the library was called")


def _calls(ctx, device):
    """Every paged call, with all that it takes on one device."""
    i32, bf = dict(dtype=torch.int32, device=device), dict(dtype=torch.bfloat16, device=device)
    P, one = cc.PagePool.empty(8, 16, 3, 4, device=device), torch.zeros(1, **i32)
    K, q, k = torch.zeros(8, 16, 2, 64, **bf), torch.zeros(1, 256, **bf), torch.zeros(1, 128, **bf)
    kv, new = cc.PagedKV(K, K.clone()), cc.NewRows(torch.zeros(2, **i32), None, 1, 1)
    return (lambda: ctx.grow_pages(P, [kv], one, one), lambda: ctx.fork_pages(P, one, one), lambda: ctx.free_pages(P, one),
            lambda: ctx.compact_pages(P, [kv]), lambda: ctx.step_paged_attention(q, new, P, kv, q.clone()),
            lambda: ctx.step_rope_append(q, k, k, new, P, kv, cc.Rope(1e4, 64), q))


def test_a_pool_on_the_host_is_refused():
    """All of it lies on one device, only not on a GPU."""
    ctx = _lib.Context.__new__(_lib.Context)
    ctx._lib, ctx._h = _NoCalls(), None
    ctx.desc = _lib.ModelDesc(64, 4, 2, 64, 64, 1e4, 1e-5, 64, 64, 64)
    for ctx._device in (None, 0, 1):
        for call in _calls(ctx, "cpu"):
            with pytest.raises(ValueError, match="context's GPU"):
                call()


@pytest.mark.gpu
def test_a_pool_of_another_gpu_is_refused():
    ctx = cc.Context(64, 4, 2, 64, 64, 1e4, 1e-5, N_cap=64, M_cap=64, T_cap=64)
    assert ctx._device == torch.cuda.current_device()
    ctx._device += 1                                        # as if it had been made there
    for call in _calls(ctx, "cuda"):
        with pytest.raises(ValueError, match="context's GPU"):
            call()
    ctx._device -= 1
    P = cc.PagePool.empty(8, 16, 3, 4)
    ctx.free_pages(P, torch.zeros(1, dtype=torch.int32, device="cuda"))
    P.len = P.len.cpu()
    with pytest.raises(ValueError, match="pool's device"):
        ctx.free_pages(P, torch.zeros(1, dtype=torch.int32, device="cuda"))
    ctx.close()


def test_numbers_that_do_not_fit_32_bits_are_refused():
    """A window of 2^32 + 5 is not one of 5."""
    big, start = (1 << 32) + 16, torch.zeros(3, dtype=torch.int32)
    for make in (lambda: cc.NewRows(start, None, big, 2), lambda: cc.NewRows(start, None, 4, big), lambda: cc.Rope(1e4, big),
                 lambda: cc.Rope(1e4, 64, scaling="turns", orig_len=1 << 31)):
        with pytest.raises(ValueError, match="32-bit"):
            make().c_struct()
    P = cc.PagePool.empty(8, 16, 3, 4, device="cpu")
    P.page_size = big
    with pytest.raises(ValueError, match="32-bit"):
        P.c_struct()
    assert cc.Rope(1e4, 64, interleaved=1 << 32).c_struct().interleaved == 1
    ctx = _lib.Context.__new__(_lib.Context)
    ctx._lib, ctx._h, ctx._device = _NoCalls(), None, -1
    ctx.desc = _lib.ModelDesc(64, 4, 2, 64, 64, 1e4, 1e-5, 64, 64, 64)
    P, K, q = cc.PagePool.empty(8, 16, 3, 4, device="cpu"), torch.zeros(8, 16, 2, 64, dtype=torch.bfloat16), torch.zeros(5, 256, dtype=torch.bfloat16)
    for kw in (dict(window=big), dict(window=5, sinks=1 << 31)):
        with pytest.raises(ValueError, match="32-bit"):
            ctx.step_paged_attention(q, cc.NewRows(start, None, 5, 5), P, cc.PagedKV(K, K), q.clone(), **kw)
