"""Arguments that the operators of residual blocks refuse, and the sizes of their workspaces (CPU: every refusal comes before any GPU call)."""
import ctypes as C

import pytest

import paper_2602_01872_amd as g


@pytest.fixture(scope="module")
def lib():
    return g.load()


P = 0x1000          # an address that is never used


def norm(lib, rows=4, width=16, x=P, ldx=16, xt=0, r=None, ldr=0, w=None, eps=1e-6, h=None, ldh=0, y=P, ldy=16, yt=0, scale=None):
    return lib.grp_rmsnorm(rows, width, x, ldx, xt, r, ldr, w, eps, h, ldh, y, ldy, yt, scale, None)


@pytest.mark.parametrize("bad,status", [
    (dict(rows=-1), g.EINVAL), (dict(width=0), g.EINVAL), (dict(width=32769, ldx=40000, ldy=40000), g.EUNSUPPORTED), (dict(x=None), g.EINVAL), (dict(y=None), g.EINVAL),
    (dict(ldx=15), g.EINVAL), (dict(ldy=15), g.EINVAL), (dict(r=P, ldr=15), g.EINVAL), (dict(h=P, ldh=15), g.EINVAL), (dict(xt=2), g.EINVAL), (dict(xt=7), g.EINVAL),
    (dict(yt=3), g.EINVAL), (dict(yt=2), g.EINVAL), (dict(eps=-1.0), g.EINVAL), (dict(eps=float("nan")), g.EINVAL), (dict(rows=1 << 32), g.EUNSUPPORTED),
    (dict(x=P + 2), g.EINVAL), (dict(y=P + 1, yt=1), g.EINVAL), (dict(w=P + 1), g.EINVAL)])
def test_norm_refuses(lib, bad, status):
    assert norm(lib, **bad) == status
    assert b"grp_rmsnorm" in lib.grp_last_error()


def test_norm_of_no_rows_is_nothing(lib):
    assert norm(lib, rows=0, x=None, y=None) == g.OK


def test_quantize_refuses(lib):
    call = lambda rows=4, width=16, x=P, ldx=16, xt=1, q=P, ldq=16, s=P: lib.grp_quantize_rows(rows, width, x, ldx, xt, q, ldq, s, None)
    for bad in (dict(rows=-1), dict(width=0), dict(x=None), dict(q=None), dict(s=None), dict(ldx=3), dict(ldq=3), dict(xt=2), dict(x=P + 1), dict(s=P + 2)):
        assert call(**bad) == g.EINVAL, bad
    assert call(rows=0) == g.OK


def test_norm_backward_refuses(lib):
    need = lib.grp_rmsnorm_backward_workspace_bytes(4, 16)
    assert need > 0 and lib.grp_rmsnorm_backward_workspace_bytes(0, 16) == 0 and lib.grp_rmsnorm_backward_workspace_bytes(4, 0) == 0

    def call(rows=4, width=16, dy=P, lddy=16, dt=0, h=P, ldh=16, ht=0, w=None, eps=1e-6, gr=None, ldg=0, dh=P, lddh=16, dw=P, ws=P, n=need):
        return lib.grp_rmsnorm_backward(rows, width, dy, lddy, dt, h, ldh, ht, w, eps, gr, ldg, dh, lddh, dw, ws, n, None)

    for bad in (dict(rows=-1), dict(width=0), dict(dy=None), dict(h=None), dict(dh=None), dict(lddy=3), dict(ldh=3), dict(lddh=3), dict(gr=P, ldg=3), dict(dt=2), dict(ht=2),
                dict(eps=-1.0), dict(dy=P + 2), dict(ws=P + 2)):
        assert call(**bad) == g.EINVAL, bad
    assert call(n=need - 1) == g.EWORKSPACE and call(ws=None) == g.EWORKSPACE


@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (16, 300, 5000), (300, 40, 8192), (4, 16, 16)])
def test_linear_refuses(lib, m, n, k):
    for e8 in (False, True):
        t = 2 if e8 else 1
        need = lib.grp_linear_workspace_bytes(g.LINEAR_FORWARD, m, n, k, t)

        def call(m=m, n=n, k=k, a=P, lda=k, w=P, ldw=k if e8 else n, t=t, a_s=None, w_s=None, b=None, act=0, r=None, ldr=0, c=P, ldc=n, ct=0, z=None, ldz=0, ws=P, size=need):
            return lib.grp_linear(m, n, k, a, lda, w, ldw, t, a_s, w_s, b, act, r, ldr, c, ldc, ct, z, ldz, ws, size, None)

        for bad in (dict(m=-1), dict(n=0), dict(k=0), dict(a=None), dict(w=None), dict(c=None), dict(lda=k - 1), dict(ldw=(k if e8 else n) - 1), dict(ldc=n - 1),
                    dict(r=P, ldr=n - 1), dict(z=P, ldz=n - 1), dict(t=0), dict(t=5), dict(act=4), dict(act=-1), dict(ct=2), dict(c=P + 2), dict(z=P + 1, ldz=n)):
            assert call(**bad) == g.EINVAL, bad
        if not e8:
            assert call(a_s=P) == g.EINVAL and call(w_s=P) == g.EINVAL and call(a=P + 1) == g.EINVAL
        if need:
            assert call(size=need - 1) == g.EWORKSPACE and call(ws=None) == g.EWORKSPACE and call(ws=P + 8) == g.EINVAL
        assert call(m=0, a=None, c=None) == g.OK


def test_linear_gradients_refuse(lib):
    m, n, k = 9, 16, 24
    dx = lambda m=m, n=n, k=k, dz=P, lddz=n, w=P, ldw=n, act=0, zin=None, ldz=0, da=P, ldda=k, dt=1: lib.grp_linear_dx(m, n, k, dz, lddz, w, ldw, act, zin, ldz, da, ldda, dt, P, 1 << 40, None)
    for bad in (dict(m=-1), dict(n=0), dict(k=0), dict(dz=None), dict(w=None), dict(da=None), dict(lddz=n - 1), dict(ldw=n - 1), dict(ldda=k - 1), dict(act=1), dict(act=9),
                dict(act=1, zin=P, ldz=k - 1), dict(dt=2), dict(dz=P + 1)):
        assert dx(**bad) == g.EINVAL, bad
    dw = lambda m=m, n=n, k=k, a=P, lda=k, dz=P, lddz=n, dw=P, lddw=n, db=None: lib.grp_linear_dw(m, n, k, a, lda, dz, lddz, dw, lddw, db, P, 1 << 40, None)
    for bad in (dict(m=-1), dict(n=0), dict(k=0), dict(a=None), dict(dz=None), dict(dw=None), dict(lda=k - 1), dict(lddz=n - 1), dict(lddw=n - 1), dict(db=P + 2), dict(a=P + 1)):
        assert dw(**bad) == g.EINVAL, bad
    big = lib.grp_linear_workspace_bytes(g.LINEAR_DW, 300_000, 64, 64, 1)
    assert big > 0 and lib.grp_linear_dw(300_000, 64, 64, P, 64, P, 64, P, 64, None, P, big - 1, None) == g.EWORKSPACE
    for bad in ((0, -1, 4, 4), (0, 4, 0, 4), (0, 4, 4, 0), (7, 4, 4, 4)):
        assert lib.grp_linear_workspace_bytes(*bad, 1) == 0


def test_gradients_refuse(lib):
    out = C.c_void_p(5)
    one = (C.c_void_p * 1)(P)
    count, kind = (C.c_int64 * 1)(4), (C.c_int32 * 1)(0)
    create = lib.grp_gradients_create
    assert create(-1, one, None, count, kind, C.byref(out)) == g.EINVAL and not out.value
    assert create(1, None, None, count, kind, C.byref(out)) == g.EINVAL
    assert create(1, one, None, None, kind, C.byref(out)) == g.EINVAL
    assert create(1, one, None, count, None, C.byref(out)) == g.EINVAL
    assert create(1, one, None, (C.c_int64 * 1)(-4), kind, C.byref(out)) == g.EINVAL
    assert create(1, one, None, count, (C.c_int32 * 1)(2), C.byref(out)) == g.EINVAL
    assert create(1, (C.c_void_p * 1)(None), None, count, kind, C.byref(out)) == g.EINVAL
    assert create(1, one, (C.c_void_p * 1)(None), count, kind, C.byref(out)) == g.EINVAL
    assert create(1, (C.c_void_p * 1)(P + 2), None, count, kind, C.byref(out)) == g.EINVAL
    assert create(1, one, None, count, kind, None) == g.EINVAL
    assert lib.grp_clip_gradients(None, 1.0, None, None) == g.EINVAL
    assert lib.grp_gradients_destroy(None) == g.OK
