"""Infinities and NaN through the layers' activations and slopes, on every way a product takes."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16
INF, NAN = float("inf"), float("nan")
# rows, columns, sums: one row, few rows, tiles of whole units and of others, W in LDS, copied operands
SIZES = [(1, 40, 16), (40, 24, 64), (300, 136, 520), (300, 137, 521), (9000, 72, 64), (9000, 71, 65), (2000, 1030, 1021)]
ACTS = ["ACT_NONE", "ACT_RELU", "ACT_GELU", "ACT_SILU"]


@pytest.fixture(scope="module")
def g():
    import paper_2602_01872_amd as lib
    lib.load()
    return lib


def value(z, act):
    """The header's formulas in 64 bits, with infinities and NaN as the arithmetic has them."""
    if act == "ACT_RELU":
        return torch.maximum(z, torch.zeros_like(z))
    if act == "ACT_GELU":
        return z * 0.5 * torch.erfc(-z * math.sqrt(0.5))
    if act == "ACT_SILU":
        return z / (1 + torch.exp(-z))
    return z


def slope(z, act):
    if act == "ACT_RELU":
        return torch.where(z.isnan(), z, (z > 0).double())
    if act == "ACT_GELU":
        return 0.5 * torch.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "ACT_SILU":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def alike(got, want, tol):
    got, want = got.double(), want.double()
    assert torch.equal(got.isnan(), want.isnan())
    inf = want.isinf()
    assert torch.equal(got[inf], want[inf]) and torch.equal(got.isinf(), inf)
    ok = want.isfinite()
    assert bool(((got - want).abs()[ok] <= tol.expand_as(want)[ok]).all())


def workspace(g, kind, m, n, k, dtype):
    b = g.grp_linear_workspace_bytes(kind, m, n, k, dtype)
    return torch.empty(b, dtype=torch.uint8, device=DEV) if b else None


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_activations(g, m, n, k, act, kind):
    """The bias brings them: column 0 infinite, 1 minus infinite, 2 NaN; A's first row brings a NaN to all columns.  A and W hold small whole numbers, so z is exact."""
    r = torch.Generator(device=DEV)
    r.manual_seed(m + n)
    e8 = kind == "e4m3"
    t = torch.float8_e4m3fn if e8 else BF16
    a = torch.randint(-1, 2, (m, k), generator=r, device=DEV).float()
    w = torch.randint(-1, 2, (k, n), generator=r, device=DEV).float() * (torch.rand(k, n, generator=r, device=DEV) < 4 / k)
    a[0, k // 2] = NAN
    bias = torch.zeros(n, device=DEV)
    bias[:3] = torch.tensor([INF, -INF, NAN])
    z64 = a.double() @ w.double() + bias.double()
    z64[0] = NAN
    aq, wq = a.to(t), (w.t().contiguous() if e8 else w).to(t)
    for ct, code in ((torch.float32, g.DTYPE_FP32), (BF16, g.DTYPE_BF16)):
        c, z = torch.full((m, n), 7.5, device=DEV, dtype=ct), torch.full((m, n), 7.5, device=DEV, dtype=BF16)
        dt = g.DTYPE_E4M3 if e8 else g.DTYPE_BF16
        g.grp_linear(m, n, k, aq, k, wq, k if e8 else n, dt, None, None, bias, getattr(g, act), None, 0, c, n, code, z, n, workspace(g, 0, m, n, k, dt))
        want = value(z64, act)
        alike(c, want, want.abs() * torch.finfo(ct).eps / 2 * 1.01 + (1 + z64.abs()) * 2.0 ** -20)
        alike(z, z64, z64.abs() * 2.0 ** -8)


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("act", ACTS[1:])
def test_slopes(g, m, n, k, act):
    """The pre-activation brings them: sizes as above, n and k in each other's place."""
    r = torch.Generator(device=DEV)
    r.manual_seed(m + n)
    dz = torch.randint(1, 3, (m, k), generator=r, device=DEV).float()
    w = (torch.rand(n, k, generator=r, device=DEV) < 4 / k).float()
    w[:, 0] = 1                                       # no sum is zero
    zin = torch.randn(m, n, generator=r, device=DEV).to(BF16)
    zin[:, 0], zin[:, 1], zin[:, 2] = INF, -INF, NAN
    lin = dz.double() @ w.double().t()
    want = lin * slope(zin.double(), act)
    for dt, code in ((torch.float32, g.DTYPE_FP32), (BF16, g.DTYPE_BF16)):
        da = torch.full((m, n), 7.5, device=DEV, dtype=dt)
        g.grp_linear_dx(m, k, n, dz.to(BF16), k, w.to(BF16), k, getattr(g, act), zin, n, da, n, code, workspace(g, 1, m, k, n, g.DTYPE_BF16))
        alike(da, want, want.abs() * torch.finfo(dt).eps / 2 * 1.01 + lin.abs() * (1 + zin.double().abs()) * 2.0 ** -20)


def norm_gradient(g, dy, h, w, eps, add=None):
    rows, width = h.shape
    dh, dw = torch.empty_like(h), torch.empty(width, device=DEV)
    ws = torch.empty(g.grp_rmsnorm_backward_workspace_bytes(rows, width), dtype=torch.uint8, device=DEV)
    code = lambda t: g.DTYPE_FP32 if t.dtype is torch.float32 else g.DTYPE_BF16
    g.grp_rmsnorm_backward(rows, width, dy, width, code(dy), h, width, code(h), w, eps, add, width, dh, width, dw, ws)
    return dh, dw


@pytest.mark.parametrize("width", [3, 8, 100, 300, 1003, 5000])
@pytest.mark.parametrize("size,eps", [(1e15, 1e-6), (1e17, 1e-6), (1e-15, 0.0), (1e-15, 1e-30), (1.0, 1e-6)])
@pytest.mark.parametrize("ht", [torch.float32, BF16])
def test_norm_gradient_of_large_and_small_rows(g, width, size, eps, ht):
    """The result is of dy / |h|'s size, which fp32 holds, though |h|^-3 is none of its numbers.  Sums of at most 48 terms a lane and tree, as everywhere: (2 x 48 + 12) 2^-24."""
    r = torch.Generator(device=DEV)
    r.manual_seed(width)
    h = (torch.randn(7, width, generator=r, device=DEV) * size).to(ht)
    dy = torch.randn(7, width, generator=r, device=DEV)
    w = 1 + 0.3 * torch.randn(width, generator=r, device=DEV)
    dh, dw = norm_gradient(g, dy, h, w, eps)
    H, U = h.double(), (dy * 1.0).double() * w.double()
    rho = 1 / torch.sqrt(H.square().mean(1, keepdim=True) + eps)
    v = H * rho
    want = rho * (U - v * (U * v).mean(1, keepdim=True))
    scale = rho * (U.abs() + v.abs() * (U * v).abs().mean(1, keepdim=True))
    assert bool(dh.isfinite().all())
    assert bool(((dh.double() - want).abs() <= want.abs() * torch.finfo(ht).eps / 2 + scale * 108 * 2.0 ** -24).all())
    assert bool(((dw.double() - (dy.double() * v).sum(0)).abs() <= (dy.double() * v).abs().sum(0) * 75 * 2.0 ** -24).all())


@pytest.mark.parametrize("width", [3, 8, 300, 5000])
def test_norm_gradient_of_rows_of_zeros(g, width):
    """rho u, and nothing else: with the smallest eps whose root is a number, too."""
    h, dy = torch.zeros(5, width, device=DEV), torch.randn(5, width, device=DEV)
    for eps in (1e-6, 1e-30, 1e-37):
        dh, dw = norm_gradient(g, dy, h, None, eps)
        want = dy.double() / math.sqrt(eps)
        assert bool(((dh.double() - want).abs() <= want.abs() * 4 * 2.0 ** -24).all()) and bool((dw == 0).all())


def test_tail_of_gelu(g):
    """Relative error of z Phi(z) below zero.  The exponent z^2 / 2 is rounded three times (2.5 2^-24 of it, 7.5e-8 z^2 of the result); the reciprocal (an ulp and a half, up
    to 2.7 times as much of the result), the exponential (an ulp), the polynomial's fit and its steps, and three products add up to less than 1.2e-6."""
    z = torch.cat([-torch.logspace(-6, 0, 2000), torch.linspace(-13, -1, 20001)]).to(DEV)
    n = z.numel()
    a, w, c = torch.zeros(1, 1, device=DEV, dtype=BF16), torch.zeros(1, n, device=DEV, dtype=BF16), torch.empty(1, n, device=DEV)
    g.grp_linear(1, n, 1, a, 1, w, n, g.DTYPE_BF16, None, None, z, g.ACT_GELU, None, 0, c, n, g.DTYPE_FP32, None, 0, workspace(g, 0, 1, n, 1, g.DTYPE_BF16))
    want = z.double() * 0.5 * torch.erfc(-z.double() * math.sqrt(0.5))
    rel = (c[0].double() / want - 1).abs()
    for lo, hi in ((0, 1), (1, 4), (4, 5), (5, 8), (8, 10), (10, 13)):
        part = (z.abs() >= lo) & (z.abs() <= hi)
        print(f"|z| {lo} .. {hi}: {float(rel[part].max()):.1e}")
    assert bool((rel <= 1.2e-6 + 7.5e-8 * z.double().square()).all())


@pytest.mark.parametrize("width", [3, 8, 40, 100, 256, 300, 1003, 3000, 5000])
@pytest.mark.parametrize("t", [torch.float32, BF16])
def test_scales_of_rows_whose_squares_vanish(g, width, t):
    """Without an eps the formula in fp32 divides by zero: y is infinite, or NaN where h is zero, and the 8-bit row's scale is y's, whatever lanes hold no column."""
    x = torch.full((3, width), 1e-30, device=DEV)
    x[1] = 0
    x[2] = 1
    x = x.to(t)
    code = g.DTYPE_FP32 if t is torch.float32 else g.DTYPE_BF16
    y, q, scale = torch.empty(3, width, device=DEV), torch.empty(3, width, device=DEV, dtype=torch.float8_e4m3fn), torch.empty(3, device=DEV)
    g.grp_rmsnorm(3, width, x, width, code, None, 0, None, 0.0, None, 0, y, width, g.DTYPE_FP32)
    g.grp_rmsnorm(3, width, x, width, code, None, 0, None, 0.0, None, 0, q, width, g.DTYPE_E4M3, scale)
    assert bool(y[0].isinf().all()) and bool(y[1].isnan().all())
    assert float(scale[0]) == INF and bool(scale[1].isnan()) and abs(float(scale[2]) * 448 - 1) < 1e-6
    assert bool(q[:2].float().isnan().all()) and bool((q[2].float() == 448).all())
