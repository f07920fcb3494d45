"""No launch of the residual-block operators holds 2^32 work-items or more, which is the limit (CPU: the rules alone are called, and refusals)."""
import ctypes as C
import os

import pytest

from tests._ways import OPS, way


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


P = 0x1000          # an address that is never used

@pytest.mark.parametrize("op", OPS)
def test_launches_of_products_hold_less_than_the_limit(lib, op):
    seen = set()
    for i in (1, 17, 64, 65, 300, 8192, 300_000, (1 << 31) - 1, 1 << 33, 1 << 40, 1 << 50):
        for j in (1, 7, 8, 47, 128, 4100, 1 << 20, 67_200_001, 67_200_008, 134_300_000, 300_000_000, (1 << 31) - 1):
            for s in (1, 8, 9, 64, 130, 500, 512, 4096, 1 << 20, 1 << 33):
                for pad, off in ((0, 0), (3, 1), (0, 8)):
                    ok, kind, _, x, y, threads = way(lib, op, i, j, s, pad, off)
                    seen.add((kind, ok))
                    if ok:
                        assert 1 <= x and x * threads < 1 << 32 and 1 <= y <= 65535, (i, j, s, kind, x, y, threads)
                    else:
                        # 2^38 results, with those that fill the tiles up: more than memory holds, or 2^31 rows or columns
                        assert kind == "tiles" and -(-i // 256) * -(-j // 256) << 16 >= 1 << 38
    assert ("tiles", True) in seen and ("tiles", False) in seen and (("few", True) in seen) == (op != "dw")


def test_few_rows_and_short_sums_of_too_many_columns_go_to_tiles(lib):
    for op in ("bf16", "e4m3", "e4m3 to fp32", "dx"):
        assert way(lib, op, 2, 134_000_000, 8)[1] == "few" and way(lib, op, 2, 134_300_000, 8)[:2] == (True, "tiles")
    assert way(lib, "bf16", 300, 67_000_001, 9)[1] == "tall" and way(lib, "bf16", 300, 67_200_001, 9)[:2] == (True, "tiles")


@pytest.mark.parametrize("m,n,k", [((1 << 31) + 1, 128, 1024), ((1 << 31) + 1, 1, 4), (1 << 40, 64, 1024), (1 << 50, 8, 2000), (70, (1 << 31) - 1, 1024)])
def test_layers_that_no_launch_holds_are_refused(lib, m, n, k):
    import paper_2602_01872_amd as g
    big = 1 << 62
    for t in (g.DTYPE_BF16, g.DTYPE_E4M3):
        s = lib.grp_linear(m, n, k, P, k, P, max(n, k), t, None, None, None, 0, None, 0, P, n, g.DTYPE_FP32, None, 0, P, big, None)
        assert s == g.EUNSUPPORTED, (t, s)
    s = lib.grp_linear_dx(m, k, n, P, k, P, max(n, k), 0, None, 0, P, n, g.DTYPE_BF16, P, big, None)
    assert s == g.EUNSUPPORTED, s
    assert b"grp_linear_dx" in lib.grp_last_error()


@pytest.mark.parametrize("n,k", [((1 << 31) - 1, (1 << 31) - 1), ((1 << 31) - 1, 4096)])
def test_gradients_of_weights_that_no_launch_holds_are_refused(lib, n, k):
    import paper_2602_01872_amd as g
    assert lib.grp_linear_dw(100, n, k, P, k, P, n, P, n, None, P, 1 << 62, None) == g.EUNSUPPORTED
