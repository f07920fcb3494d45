"""Outputs in the place of inputs whose rows lie at other distances are refused: they overlap other rows (CPU: before any GPU call)."""
import pytest

import paper_2602_01872_amd as g

P, Q, R = 0x1000, 0x2000, 0x3000          # addresses that are never used
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return g.load()


def refused(lib, status, name):
    return status == g.EINVAL and name in lib.grp_last_error() and b"in place of" in lib.grp_last_error()


def test_norm(lib):
    call = lambda rows=4, ldx=16, r=None, ldr=16, h=None, ldh=16, y=Q, ldy=16, yt=0: lib.grp_rmsnorm(rows, 16, P, ldx, 0, r, ldr, None, 1e-6, h, ldh, y, ldy, yt, None, None)
    assert refused(lib, call(h=P, ldh=17), b"grp_rmsnorm")
    assert refused(lib, call(h=P, ldx=20), b"grp_rmsnorm")
    assert refused(lib, call(r=R, h=R, ldr=18), b"grp_rmsnorm")
    assert not refused(lib, call(h=P), b"grp_rmsnorm") and not refused(lib, call(rows=1, h=P, ldh=17), b"grp_rmsnorm")
    assert not refused(lib, call(r=R, h=R, ldr=18, ldh=18), b"grp_rmsnorm")


def test_norm_gradient(lib):
    need = lib.grp_rmsnorm_backward_workspace_bytes(4, 16)
    call = lambda ldh=16, gr=None, ldg=16, dh=P, lddh=16: lib.grp_rmsnorm_backward(4, 16, Q, 16, 0, P, ldh, 0, None, 1e-6, gr, ldg, dh, lddh, None, None, need, None)
    assert refused(lib, call(lddh=17), b"grp_rmsnorm_backward") and refused(lib, call(ldh=17), b"grp_rmsnorm_backward")
    assert refused(lib, call(gr=R, dh=R, ldg=17), b"grp_rmsnorm_backward")
    assert not refused(lib, call(), b"grp_rmsnorm_backward") and not refused(lib, call(gr=R, dh=R, ldg=17, lddh=17), b"grp_rmsnorm_backward")


@pytest.mark.parametrize("m,n,k", [(4, 16, 24), (300, 40, 64), (9000, 64, 64)])
def test_linear(lib, m, n, k):
    call = lambda m=m, r=None, ldr=n, c=R, ldc=n: lib.grp_linear(m, n, k, P, k, Q, n, g.DTYPE_BF16, None, None, None, 0, r, ldr, c, ldc, g.DTYPE_BF16, None, 0, P, BIG, None)
    assert refused(lib, call(r=R, ldr=n + 1), b"grp_linear") and refused(lib, call(r=R, ldc=n + 8), b"grp_linear")
    assert not refused(lib, call(r=R), b"grp_linear") and not refused(lib, call(r=P, ldr=n + 1), b"grp_linear") and not refused(lib, call(m=1, r=R, ldr=n + 1), b"grp_linear")
