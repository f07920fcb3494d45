"""No launch of the residual-block operators holds 2^32 work-items or more, which is the limit (CPU: the rules alone are called, and refusals)."""
import ctypes as C
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2602_01872_amd as g
    if not os.path.exists(g.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return g.load()


@pytest.mark.parametrize("lanes", [8, 16, 32, 64, 256, 1024])
def test_rows_of_a_norm_fit_a_launch(lib, lanes):
    fn = getattr(lib, "_ZN3grp19norm_rows_of_launchEi")        # int64_t grp::norm_rows_of_launch(int lanes)
    fn.argtypes, fn.restype = [C.c_int], C.c_int64
    rows, threads = fn(lanes), max(256, lanes)
    per = threads // lanes
    assert rows > 0 and rows % per == 0
    assert rows // per * threads < 1 << 32 and (rows + 1) * lanes <= 1 << 32
    assert rows >= (1 << 21)                                   # and large launches stay one
