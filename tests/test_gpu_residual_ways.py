"""Linear layers on every way that a product takes, against 64 bits, with bounds that see a lost part of a sum (``sum_error``): on each result, and on the norm of
the error of all of them.  bf16 results of e4m3 products: 7 2^-13 of the sum of the terms' sizes more on a result, 2^-12 of the root of the sum of their squares on the
norm (of eight products seven are cut by up to 2^-13 of the largest, with either sign).  Activations: 2^-20 of 1 + |z|, and at most 1.2 times z's error."""
import math

import pytest
import torch

from tests._ways import WAYS, sum_error

pytestmark = pytest.mark.gpu
DEV = "cuda"
FP32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
NAN = float("nan")


@pytest.fixture(scope="module")
def g():
    import paper_2602_01872_amd as lib
    lib.load()
    yield lib
    torch.cuda.empty_cache()


class Mat:
    """rows x cols, `pad` elements between rows and `off` before the first; what is around them is NaN."""

    def __init__(self, rows, cols, dtype, pad, off, value=None):
        self.ld = cols + pad
        self.buf = torch.empty(off + rows * self.ld + 64, device=DEV, dtype=dtype)
        self.bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[self.buf.element_size()]
        self.buf.view(self.bits).fill_(-1 if self.bits is not torch.uint8 else 255)       # NaN in every type
        self.at = lambda t: t[off:off + rows * self.ld].view(rows, self.ld)[:, :cols]
        self.v = self.at(self.buf)
        if value is not None:
            self.at(self.buf.view(self.bits)).copy_(value.to(dtype).view(self.bits))

    def data_ptr(self):
        return self.v.data_ptr()

    def untouched(self):
        around = self.buf.view(self.bits).clone()
        self.at(around).fill_(-1 if self.bits is not torch.uint8 else 255)
        return bool((around == (-1 if self.bits is not torch.uint8 else 255)).all())


def draw(r, rows, cols, scale=1.0):
    return torch.randn(rows, cols, generator=r, device=DEV) * scale


def half(t):
    return torch.finfo(t).eps / 2


def act64(z, act):
    if act == "ACT_RELU":
        return z.clamp_min(0)
    if act == "ACT_GELU":
        return z * 0.5 * torch.erfc(-z * math.sqrt(0.5))
    if act == "ACT_SILU":
        return z * torch.sigmoid(z)
    return z


def slope64(z, act):
    if act == "ACT_RELU":
        return (z > 0).double()
    if act == "ACT_GELU":
        return 0.5 * torch.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "ACT_SILU":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def check(got, want, each, norm, t):
    """each: what every result may be off by before it is rounded to t; norm: the norm of the error."""
    off = got.double() - want
    bad = ~(off.abs() <= each + (want.abs() + each) * half(t))
    assert not bool(bad.any()), (int(bad.sum()), float(off.abs().nan_to_num(1e30).max()))
    assert float(off.norm()) <= norm + (float(want.norm()) + norm) * half(t)


def room(g, kind, m, n, k, dtype):
    b = g.grp_linear_workspace_bytes(kind, m, n, k, dtype)
    return torch.full((b,), 255, dtype=torch.uint8, device=DEV) if b else None           # NaN


def forward(g, op, m, n, k, pad, off):
    e8 = op != "bf16"
    et, code = (E4M3, g.DTYPE_E4M3) if e8 else (BF16, g.DTYPE_BF16)
    r = torch.Generator(device=DEV)
    r.manual_seed(m + 3 * n + 7 * k)
    A, W = draw(r, m, k).to(et).float(), draw(r, k, n, 1.0 if e8 else k ** -0.5).to(et).float()
    a, w = Mat(m, k, et, pad, off, A), Mat(n, k, et, pad, off, W.t().contiguous()) if e8 else Mat(k, n, et, pad, off, W)
    a_s = torch.rand(m, generator=r, device=DEV) + 0.1 if e8 else None
    w_s = (torch.rand(n, generator=r, device=DEV) + 0.1) * k ** -0.5 if e8 else None
    bias, res = torch.randn(n, generator=r, device=DEV), draw(r, m, n)
    A, W = A.double(), W.double()
    if e8:
        A, W = A * a_s.double()[:, None], W * w_s.double()
    z64 = A @ W + bias.double()
    size = (A.square() @ W.square()).sqrt()
    types = {"bf16": (FP32, BF16), "e4m3": (BF16,), "e4m3 to fp32": (FP32,)}[op]
    for ct in types:
        each, norm = size * 6 * sum_error(k), float(size.norm()) * sum_error(k)
        if op == "e4m3":
            each, norm = each + (A.abs() @ W.abs()) * 7 * 2.0 ** -13, norm + float(size.norm()) * 2.0 ** -12
        each = each + (z64.abs() + bias.double().abs()) * 4 * 2.0 ** -24                   # the scales and the bias, rounded
        norm = norm + (float(z64.norm()) + float(bias.double().norm()) * m ** 0.5) * 4 * 2.0 ** -24
        for act, plain in (("ACT_GELU" if ct is BF16 else "ACT_SILU", False), ("ACT_NONE", True)):
            rr = Mat(m, n, ct, pad, off, res)
            c, z = Mat(m, n, ct, pad, off), Mat(m, n, BF16, pad, off)
            g.grp_linear(m, n, k, a, a.ld, w, w.ld, code, a_s, w_s, bias, getattr(g, act), None if plain else rr, rr.ld, c, c.ld,
                         g.DTYPE_FP32 if ct is FP32 else g.DTYPE_BF16, None if plain else z, z.ld, room(g, g.LINEAR_FORWARD, m, n, k, code))
            want = act64(z64, act)
            more = torch.zeros_like(z64) if plain else (1 + z64.abs()) * 2.0 ** -20 + (want.abs() + rr.v.double().abs()) * 2.0 ** -23
            if not plain:
                want = want + rr.v.double()
                check(z.v, z64, each, norm, BF16)
            check(c.v, want, (1 if plain else 1.2) * each + more, (1 if plain else 1.2) * norm + float(more.norm()), ct)
            assert c.untouched() and z.untouched() and (not plain or bool(z.v.isnan().all()))


def by_input(g, m, k, n, pad, off):
    """m x k results, sums of n."""
    r = torch.Generator(device=DEV)
    r.manual_seed(m + 3 * n + 7 * k)
    dz, w = Mat(m, n, BF16, pad, off, draw(r, m, n)), Mat(k, n, BF16, pad, off, draw(r, k, n, n ** -0.5))
    zin = Mat(m, k, BF16, pad, off, draw(r, m, k))
    P, Q, Z = dz.v.double(), w.v.double(), zin.v.double()
    lin, size = P @ Q.t(), (P.square() @ Q.square().t()).sqrt()
    for act, dt in (("ACT_GELU", BF16), ("ACT_RELU", FP32), ("ACT_NONE", BF16)):
        da = Mat(m, k, dt, pad, off)
        none = act == "ACT_NONE"
        g.grp_linear_dx(m, n, k, dz, dz.ld, w, w.ld, getattr(g, act), None if none else zin, zin.ld, da, da.ld, g.DTYPE_FP32 if dt is FP32 else g.DTYPE_BF16,
                        room(g, g.LINEAR_DX, m, n, k, g.DTYPE_BF16))
        slope = slope64(Z, act)
        more = lin.abs() * (1 + Z.abs()) * 2.0 ** -20 if act == "ACT_GELU" else torch.zeros_like(lin)
        check(da.v, lin * slope, size * slope.abs() * 6 * sum_error(n) + more, float((size * slope).norm()) * sum_error(n) + float(more.norm()), dt)
        assert da.untouched()


def by_weight(g, k, n, m, pad, off):
    """k x n results, sums of m rows."""
    r = torch.Generator(device=DEV)
    r.manual_seed(m + 3 * n + 7 * k)
    a, dz = Mat(m, k, BF16, pad, off, draw(r, m, k)), Mat(m, n, BF16, pad, off, draw(r, m, n))
    A, D = a.v.double(), dz.v.double()
    want, size = A.t() @ D, (A.square().t() @ D.square()).sqrt()
    for sums in (True, False):
        dw, db = Mat(k, n, FP32, pad, off), torch.full((n + 2,), -3.0, device=DEV)
        g.grp_linear_dw(m, n, k, a, a.ld, dz, dz.ld, dw, dw.ld, db if sums else None, room(g, g.LINEAR_DW, m, n, k, g.DTYPE_BF16))
        check(dw.v, want, size * 6 * sum_error(m), float(size.norm()) * sum_error(m), FP32)
        if sums:
            columns = D.square().sum(0).sqrt()
            check(db[:n], D.sum(0), columns * 6 * sum_error(m), float(columns.norm()) * sum_error(m), FP32)
        assert dw.untouched() and bool((db[n if sums else 0:] == -3).all())


@pytest.mark.parametrize("op,i,j,s,pad,off", [(op, *e) for op in WAYS for e in WAYS[op]])
def test_way(g, op, i, j, s, pad, off):
    if op == "dx":
        by_input(g, i, j, s, pad, off)
    elif op == "dw":
        by_weight(g, i, j, s, pad, off)
    else:
        forward(g, op, i, j, s, pad, off)


def test_rows_that_begin_past_32_bits(g):
    """2.3e9 elements of A: sums over all rows, first and last columns of the result, and first and last rows of the forward product."""
    m, k, n = 140_001, 16_384, 16
    r = torch.Generator(device=DEV)
    r.manual_seed(1)
    a = torch.empty(m, k, device=DEV, dtype=BF16)
    for i in range(0, m, 20_000):
        a[i:i + 20_000] = torch.randn(min(20_000, m - i), k, generator=r, device=DEV)
    dz, w = draw(r, m, n).to(BF16), draw(r, k, n, k ** -0.5).to(BF16)
    dw, c = torch.empty(k, n, device=DEV), torch.empty(m, n, device=DEV)
    g.grp_linear_dw(m, n, k, a, k, dz, n, dw, n, None, room(g, g.LINEAR_DW, m, n, k, g.DTYPE_BF16))
    for at in (slice(0, 64), slice(8192, 8256), slice(k - 64, k)):
        A, D = a[:, at].double(), dz.double()
        size = (A.square().t() @ D.square()).sqrt()
        check(dw[at], A.t() @ D, size * 6 * sum_error(m), float(size.norm()) * sum_error(m), FP32)
    g.grp_linear(m, n, k, a, k, w, n, g.DTYPE_BF16, None, None, None, g.ACT_NONE, None, 0, c, n, g.DTYPE_FP32, None, 0, room(g, g.LINEAR_FORWARD, m, n, k, g.DTYPE_BF16))
    for at in (slice(0, 300), slice(131_000, 131_300), slice(m - 300, m)):
        A, W = a[at].double(), w.double()
        size = (A.square() @ W.square()).sqrt()
        check(c[at], A @ W, size * 6 * sum_error(k), float(size.norm()) * sum_error(k), FP32)
