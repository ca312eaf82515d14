"""More checks of the paged calls' arguments (csrc/paged_plan.h), compiled by the host compiler and asked without a GPU."""
import ctypes as C
import subprocess

import pytest

from paper_2510_10129_amd import build
from paper_2510_10129_amd._lib import CC_ERR_NULL, CC_ERR_SHAPE, CC_OK, _Pool

from test_paged_plan import A, CXX, _pool

SHIM = r"""
#include "paged_plan.h"
extern "C" {
int pool(const cc_page_pool* p) { return cc_check_pool(p).code; }
int grow(const cc_page_pool* p, const int32_t* status) { return cc_check_grow(*p, status).code; }
int pool_size() { return sizeof(cc_page_pool); }
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
