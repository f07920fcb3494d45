"""Lists of a gradient's tensors that no memory holds are refused before a list of their pieces is made (CPU: before any GPU call)."""
import ctypes as C

import pytest

import paper_2602_01872_amd as g

P = 0x1000          # an address that is never used


@pytest.mark.parametrize("counts", [[1 << 44], [1 << 62], [1 << 62] * 4, [(1 << 63) - 1] * 3, [1 << 39] * 40])
@pytest.mark.parametrize("kind", [0, 1])
def test_too_many_elements(counts, kind):
    lib = g.load()
    n = len(counts)
    out = C.c_void_p(5)
    s = lib.grp_gradients_create(n, (C.c_void_p * n)(*[P] * n), None, (C.c_int64 * n)(*counts), (C.c_int32 * n)(*[kind] * n), C.byref(out))
    assert s == g.EUNSUPPORTED and not out.value
    assert b"grp_gradients_create" in lib.grp_last_error()
