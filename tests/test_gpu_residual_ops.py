"""Operators of residual blocks (norm, 8-bit rows, linear layers, clipping) against plain implementations in 64 bits, at the sizes where
they can go wrong: one row and one column, widths around the units of 16 bytes and around the tiles, rows that start at any element, rows of
zeros, infinities and NaN, outputs in place, other streams and graph replays.

Tolerances: a rounding to type t is off by at most eps(t) / 2 of the value; fp32 sums of n terms by (n + a few) 2^-24 of the sum of the terms'
sizes; the matrix unit also cuts (twice that); activations are evaluated to 2^-20 of (1 + |z|).  bf16 results of e4m3 products are made by the 8-bit
matrix instructions, which cut seven products of every eight below 2^-13 of the largest: 7 2^-13 of the sum of the terms' sizes more."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
FP32, BF16 = torch.float32, torch.bfloat16
CODE = {}


@pytest.fixture(scope="module")
def g():
    import paper_2602_01872_amd as lib
    lib.load()
    CODE.update({FP32: lib.DTYPE_FP32, BF16: lib.DTYPE_BF16, torch.float8_e4m3fn: lib.DTYPE_E4M3})
    return lib


def half_step(t):
    return torch.finfo(t).eps / 2


def gen(seed):
    r = torch.Generator(device=DEV)
    r.manual_seed(seed)
    return r


class Mat:
    """rows x cols of pitch cols + pad, `off` elements into an allocation whose other elements are NaN."""

    def __init__(self, rows, cols, dtype, pad=0, off=0, value=None):
        self.rows, self.cols, self.ld = rows, cols, cols + pad
        self.buf = torch.full((off + rows * self.ld + 64,), float("nan"), device=DEV).to(dtype)
        self.v = self.buf[off:off + rows * self.ld].view(rows, self.ld)[:, :cols]
        if value is not None:
            self.v.copy_(value)
        self.outside = torch.ones_like(self.buf, dtype=torch.bool)
        self.outside[off:off + rows * self.ld].view(rows, self.ld)[:, :cols] = False

    def data_ptr(self):
        return self.v.data_ptr()

    def d(self):
        return self.v.double()

    def untouched(self):
        return bool(self.buf.float()[self.outside].isnan().all())


def randn(rows, cols, r, scale=1.0):
    return torch.randn(rows, cols, generator=r, device=DEV) * scale


def within(got, want, tol):
    got, want = got.double(), want.double()
    bad = ~((got - want).abs() <= tol)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, worst {float(((got - want).abs() - tol).nan_to_num(1e30).max())}"


# ------------------------------------------------------------------------------------------------ norm
WIDTHS = [1, 3, 4, 5, 7, 8, 9, 15, 16, 33, 64, 65, 127, 250, 256, 257, 511, 515, 1003, 1025, 2047, 2056, 4099, 8192, 8201, 16390, 32768]


def seq(width):
    return 32 + 16                     # terms that a lane adds one after another (at most 32), and the tree over lanes and wavefronts


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("xt,yt", [(FP32, FP32), (FP32, BF16), (BF16, FP32), (BF16, BF16)])
def test_norm(g, width, xt, yt):
    for rows, pad, off, residual, keep, wt in [(1, 0, 0, True, True, True), (5, 3, 1, True, False, True), (67, 1, 3, False, True, False), (33, 8, 0, True, True, True)]:
        r = gen(width * 7 + rows)
        x, a = Mat(rows, width, xt, pad, off, randn(rows, width, r)), Mat(rows, width, xt, pad, off, randn(rows, width, r, 3.0))
        h, y = Mat(rows, width, xt, pad, off), Mat(rows, width, yt, pad, off)
        w = 1 + 0.3 * torch.randn(width, generator=r, device=DEV)
        g.grp_rmsnorm(rows, width, x, x.ld, CODE[xt], a if residual else None, a.ld, w if wt else None, 1e-5, h if keep else None, h.ld, y, y.ld, CODE[yt])
        want_h = x.d() + (a.d() if residual else 0)
        want_y = want_h / torch.sqrt(want_h.square().mean(1, keepdim=True) + 1e-5) * (w.double() if wt else 1)
        within(y.v, want_y, want_y.abs() * (half_step(yt) + (seq(width) + 8) * U))
        if keep:
            within(h.v, want_h, want_h.abs() * (half_step(xt) + U))
        else:
            assert bool(h.v.isnan().all())
        assert y.untouched() and h.untouched() and x.untouched()


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("xt", [FP32, BF16])
@pytest.mark.parametrize("normalise", [True, False])
def test_eight_bit_rows(g, width, xt, normalise):
    for rows, pad, off in [(1, 0, 0), (35, 3, 1), (9, 16, 0)]:
        r = gen(width * 3 + rows)
        x = Mat(rows, width, xt, pad, off, randn(rows, width, r) * torch.exp(2 * randn(rows, 1, r)))
        if rows > 4:
            x.v[2] = 0
            x.v[3] *= 1e-30
        q, scale = Mat(rows, width, torch.float8_e4m3fn, pad, off), torch.full((rows + 1,), -7.0, device=DEV)
        w = 1 + 0.3 * torch.randn(width, generator=r, device=DEV)
        if normalise:
            g.grp_rmsnorm(rows, width, x, x.ld, CODE[xt], None, 0, w, 1e-5, None, 0, q, q.ld, g.DTYPE_E4M3, scale)
            y = x.d() / torch.sqrt(x.d().square().mean(1, keepdim=True) + 1e-5) * w.double()
        else:
            g.grp_quantize_rows(rows, width, x, x.ld, CODE[xt], q, q.ld, scale)
            y = x.d()
        s = scale[:rows].double()
        want_s = (y.abs().amax(1) / 448).clamp_min(2.0 ** -126)
        within(s, want_s, want_s * (seq(width) + 10) * U)
        assert float(scale[rows]) == -7.0 and q.untouched()
        got = q.v.float().double() * s[:, None]
        within(got, y, y.abs() * (2.0 ** -4 + (seq(width) + 10) * U) + s[:, None] * 2.0 ** -10)
        full = q.v.float().abs().amax(1)
        assert bool((full[y.abs().amax(1) > 448 * 2.0 ** -126] == 448).all())          # the largest element takes the whole range


def test_eight_bit_values_are_the_nearest(g):
    """Every quotient that is no tie goes to the nearest e4m3 number: checked by the distance to all 256 of them."""
    r = gen(5)
    x = randn(64, 1000, r)
    q, scale = torch.empty(64, 1000, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(64, device=DEV)
    g.grp_quantize_rows(64, 1000, x, 1000, g.DTYPE_FP32, q, 1000, scale)
    numbers = torch.arange(256, device=DEV, dtype=torch.uint8).view(torch.float8_e4m3fn).float().double()
    numbers = numbers[numbers.isfinite()]
    v = x.double() / scale.double()[:, None]
    nearest = torch.stack([(v[i:i + 1].T - numbers).abs().amin(1) for i in range(64)])
    off = (q.float().double() - v).abs()
    assert bool((off <= nearest + v.abs() * 4 * U).all())


def test_norm_of_special_rows(g):
    """Zeros, infinities, NaN and squares past fp32: as the fp32 formula has them, and no row touches another."""
    inf, nan = float("inf"), float("nan")
    for width in (8, 100, 300, 3000):
        x = torch.ones(7, width, device=DEV)
        x[1] = 0
        x[2, width // 2] = inf
        x[3, width - 1] = -inf
        x[4, 0] = nan
        x[5] = 1e30
        for t in (FP32, BF16):
            xs = x.to(t)
            y = torch.empty(7, width, device=DEV)
            g.grp_rmsnorm(7, width, xs, width, CODE[t], None, 0, None, 1e-6, None, 0, y, width, g.DTYPE_FP32)
            h = xs.float()
            want = h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-6)
            assert torch.allclose(y, want, rtol=1e-5, atol=0, equal_nan=True)
            q, s = torch.empty(7, width, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(7, device=DEV)
            g.grp_quantize_rows(7, width, xs, width, CODE[t], q, width, s)
            want_s = (h.abs().amax(1) / 448).clamp_min(2.0 ** -126)
            assert torch.equal(s.isnan(), want_s.isnan()) and torch.equal(s.nan_to_num(1.0), want_s.nan_to_num(1.0))
            assert torch.equal(q.float().nan_to_num(7.0), (h / s[:, None]).to(torch.float8_e4m3fn).float().nan_to_num(7.0))


@pytest.mark.parametrize("width", [3, 8, 100, 256, 1003, 4099])
def test_norm_in_place(g, width):
    rows = 41
    r = gen(width)
    for t in (FP32, BF16):
        x, a = randn(rows, width, r).to(t), randn(rows, width, r).to(t)
        outs = []
        for place in ("apart", "x", "r"):
            xi, ai, y = x.clone(), a.clone(), torch.empty(rows, width, device=DEV, dtype=BF16)
            h = {"apart": torch.empty_like(x), "x": xi, "r": ai}[place]
            g.grp_rmsnorm(rows, width, xi, width, CODE[t], ai, width, None, 1e-6, h, width, y, width, g.DTYPE_BF16)
            outs.append((h, y))
        for h, y in outs[1:]:
            assert torch.equal(h, outs[0][0]) and torch.equal(y, outs[0][1])


def norm_grad64(dy, h, w, eps, add):
    width = h.shape[1]
    rho = 1 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    u = dy * w
    k = rho ** 3 * (u * h).mean(1, keepdim=True)
    k_size = rho ** 3 * (u * h).abs().mean(1, keepdim=True)
    dh = rho * u - h * k + add
    size = (rho * u).abs() + h.abs() * k_size + (add.abs() if torch.is_tensor(add) else 0)
    return dh, size, (dy * h * rho).sum(0), (dy * h * rho).abs().sum(0)


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dt,ht", [(FP32, FP32), (BF16, FP32), (FP32, BF16), (BF16, BF16)])
def test_norm_gradient(g, width, dt, ht):
    for rows, pad, off, residual, wt in [(1, 0, 0, True, True), (70, 3, 1, True, True), (133, 8, 0, False, False)]:
        r = gen(width + rows)
        dy, h = Mat(rows, width, dt, pad, off, randn(rows, width, r)), Mat(rows, width, ht, pad, off, randn(rows, width, r, 2.0))
        add, dh = Mat(rows, width, ht, pad, off, randn(rows, width, r)), Mat(rows, width, ht, pad, off)
        w = 1 + 0.3 * torch.randn(width, generator=r, device=DEV)
        dw = torch.full((width + 3,), -5.0, device=DEV)
        ws = torch.empty(g.grp_rmsnorm_backward_workspace_bytes(rows, width), dtype=torch.uint8, device=DEV)
        g.grp_rmsnorm_backward(rows, width, dy, dy.ld, CODE[dt], h, h.ld, CODE[ht], w if wt else None, 1e-5, add if residual else None, add.ld, dh, dh.ld, dw, ws)
        want, size, want_w, size_w = norm_grad64(dy.d(), h.d(), w.double() if wt else 1.0, 1e-5, add.d() if residual else 0.0)
        within(dh.v, want, want.abs() * half_step(ht) + size * (2 * seq(width) + 12) * U)
        within(dw[:width], want_w, size_w * (rows + seq(width) + 12) * U)
        assert dh.untouched() and bool((dw[width:] == -5).all())
        # without the weight's gradient: no workspace, the same dh; in place of g, and of h
        for place in ("apart", "g", "h"):
            hi, ai = Mat(rows, width, ht, pad, off, h.v), Mat(rows, width, ht, pad, off, add.v)
            out = {"apart": Mat(rows, width, ht, pad, off), "g": ai, "h": hi}[place]
            g.grp_rmsnorm_backward(rows, width, dy, dy.ld, CODE[dt], hi, h.ld, CODE[ht], w if wt else None, 1e-5, ai if residual else None, add.ld, out, out.ld,
                                   None, None)
            assert torch.equal(out.v, dh.v)


def test_norm_gradient_against_differences(g):
    rows, width = 6, 37
    r = gen(9)
    h, dy, w = randn(rows, width, r), randn(rows, width, r), 1 + 0.3 * torch.randn(width, generator=r, device=DEV)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    ws = torch.empty(g.grp_rmsnorm_backward_workspace_bytes(rows, width), dtype=torch.uint8, device=DEV)
    g.grp_rmsnorm_backward(rows, width, dy, width, 0, h, width, 0, w, 1e-5, None, 0, dh, width, dw, ws)

    def loss(hh, ww):
        return (hh / torch.sqrt(hh.square().mean(1, keepdim=True) + 1e-5) * ww * dy.double()).sum()

    step = 1e-5                # central differences in 64 bits: their own error is step^2 and 2^-52 / step, both below 1e-9 here
    for i, c in [(0, 0), (1, 36), (3, 17), (5, 4)]:
        e = torch.zeros(rows, width, device=DEV, dtype=torch.float64)
        e[i, c] = step
        diff = (loss(h.double() + e, w.double()) - loss(h.double() - e, w.double())) / (2 * step)
        assert abs(float(dh[i, c]) - float(diff)) < 1e-5
        e1 = torch.zeros(width, device=DEV, dtype=torch.float64)
        e1[c] = step
        diff = (loss(h.double(), w.double() + e1) - loss(h.double(), w.double() - e1)) / (2 * step)
        assert abs(float(dw[c]) - float(diff)) < 1e-5


def test_no_rows(g):
    x, w, dw = torch.empty(0, 16, device=DEV), torch.ones(16, device=DEV), torch.full((16,), 3.0, device=DEV)
    g.grp_rmsnorm(0, 16, x, 16, 0, None, 0, w, 1e-6, None, 0, x, 16, 0)
    g.grp_quantize_rows(0, 16, x, 16, 0, x, 16, x)
    g.grp_rmsnorm_backward(0, 16, x, 16, 0, x, 16, 0, w, 1e-6, None, 0, x, 16, dw, None)
    assert bool((dw == 0).all())
    b = torch.empty(0, 8, device=DEV, dtype=BF16)
    wt = torch.ones(8, 16, device=DEV, dtype=BF16)
    g.grp_linear(0, 16, 8, b, 8, wt, 16, g.DTYPE_BF16, None, None, None, g.ACT_NONE, None, 0, x, 16, 0, None, 0, None)
    g.grp_linear_dx(0, 16, 8, b, 16, wt, 16, g.ACT_NONE, None, 0, b, 8, g.DTYPE_BF16, None)
    dwt, db = torch.ones(8, 16, device=DEV), torch.ones(16, device=DEV)
    n = g.grp_linear_workspace_bytes(g.LINEAR_DW, 0, 16, 8, g.DTYPE_BF16)
    g.grp_linear_dw(0, 16, 8, b, 8, b, 16, dwt, 16, db, torch.empty(n, dtype=torch.uint8, device=DEV) if n else None)
    assert bool((dwt == 0).all()) and bool((db == 0).all())


# ------------------------------------------------------------------------------------------------ linear
# M, N, K: single rows and columns, around tiles and steps, long sums, many rows
SHAPES = [(1, 1, 1), (1, 8, 8), (1, 256, 256), (1, 130, 1000), (2, 1003, 77), (7, 64, 64), (16, 128, 512), (17, 129, 131), (33, 48, 4100), (64, 64, 8), (100, 300, 64),
          (127, 255, 129), (128, 128, 128), (130, 260, 200), (255, 72, 1024), (257, 513, 96), (300, 8, 2000), (513, 1030, 250), (1000, 40, 31), (3001, 256, 256),
          (5000, 17, 9), (700, 700, 700)]
ACTS = ["none", "relu", "gelu", "silu"]


def act64(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z * math.sqrt(0.5))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def slope64(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * torch.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def code(g, act):
    return {"none": g.ACT_NONE, "relu": g.ACT_RELU, "gelu": g.ACT_GELU, "silu": g.ACT_SILU}[act]


def workspace(g, kind, m, n, k, dtype):
    b = g.grp_linear_workspace_bytes(kind, m, n, k, dtype)
    return torch.full((b,), 255, dtype=torch.uint8, device=DEV) if b else None      # NaN


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("e8", [False, True])
def test_linear(g, m, n, k, e8):
    variants = [(0, 0, FP32, "none", False, False, False), (8, 0, BF16, "gelu", True, True, True), (3, 1, FP32, "silu", True, True, True),
                (16, 0, BF16, "relu", True, True, False), (1, 3, BF16, "none", False, False, True)]
    for pad, off, ct, act, residual, bias, keep in variants:
        r = gen(m * 31 + n * 7 + k + pad)
        et = torch.float8_e4m3fn if e8 else BF16
        a = Mat(m, k, et, pad, off, randn(m, k, r).to(et))
        w = Mat(n, k, et, pad, off, randn(n, k, r, k ** -0.5 if not e8 else 1.0).to(et)) if e8 else Mat(k, n, et, pad, off, randn(k, n, r, k ** -0.5).to(et))
        scaled = e8 and residual
        a_s = torch.rand(m, generator=r, device=DEV) + 0.1 if scaled else None
        w_s = (torch.rand(n, generator=r, device=DEV) + 0.1) * k ** -0.5 if scaled else None
        b = torch.randn(n, generator=r, device=DEV) if bias else None
        res = Mat(m, n, ct, pad, off, randn(m, n, r))
        c, z = Mat(m, n, ct, pad, off), Mat(m, n, BF16, pad, off)
        ws = workspace(g, g.LINEAR_FORWARD, m, n, k, CODE[et])
        g.grp_linear(m, n, k, a, a.ld, w, w.ld, CODE[et], a_s, w_s, b, code(g, act), res if residual else None, res.ld, c, c.ld, CODE[ct], z if keep else None, z.ld, ws)
        W = w.v.float().double().t() if e8 else w.d()
        A = a.v.float().double()
        if scaled:
            W, A = W * w_s.double(), A * a_s.double()[:, None]
        lin = A @ W
        z64 = lin + (b.double() if bias else 0)
        off_z = (A.abs() @ W.abs()) * (k + 12) * 2 * U + z64.abs() * 4 * U + (b.double().abs() * U if bias else 0)
        if e8 and ct is BF16:
            off_z = off_z + (A.abs() @ W.abs()) * 7 * 2.0 ** -13
        want = act64(z64, act) + (res.d() if residual else 0)
        tol = 1.2 * off_z + (0 if act == "none" else (1 + z64.abs()) * 2.0 ** -20) + want.abs() * (half_step(ct) + 2 * U) + (res.d().abs() * 2 * U if residual else 0)
        within(c.v, want, tol * (1 + half_step(ct)))
        assert float((c.d() - want).norm()) <= float(want.norm()) * (half_step(ct) + 2.0 ** -13)
        if keep:
            within(z.v, z64, (off_z + z64.abs() * half_step(BF16)) * 1.01)
        else:
            assert bool(z.v.isnan().all())
        assert c.untouched() and z.untouched()
        if residual:                                                   # C in place of r
            c2 = Mat(m, n, ct, pad, off, res.v)
            g.grp_linear(m, n, k, a, a.ld, w, w.ld, CODE[et], a_s, w_s, b, code(g, act), c2, c2.ld, c2, c2.ld, CODE[ct], None, 0, ws)
            assert torch.equal(c2.v, c.v)


# sizes at which the other ways are taken: W kept in LDS (short sums, several groups of columns, rows at odd elements), copies as whole units, large tiles
MORE_SHAPES = [(9000, 700, 60), (8200, 90, 300), (8193, 130, 257), (2000, 1030, 1021), (9000, 300, 515), (3000, 1001, 900), (6000, 2600, 136), (70, 520, 248), (12000, 61, 8),
               (65, 9, 9)]


@pytest.mark.parametrize("m,n,k", MORE_SHAPES)
def test_linear_other_ways(g, m, n, k):
    test_linear(g, m, n, k, False)
    test_linear(g, m, n, k, True)
    test_linear_dx(g, m, k, n)
    test_linear_dw(g, m, n, k)


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_linear_dx(g, m, n, k):
    for i, (pad, off, dt) in enumerate([(0, 0, FP32), (8, 0, BF16), (3, 1, BF16), (1, 0, FP32)]):
        act = ACTS[i]
        r = gen(m + n * 5 + k * 3 + pad)
        dz, w = Mat(m, n, BF16, pad, off, randn(m, n, r)), Mat(k, n, BF16, pad, off, randn(k, n, r, n ** -0.5))
        zin, da = Mat(m, k, BF16, pad, off, randn(m, k, r, 2.0)), Mat(m, k, dt, pad, off)
        ws = workspace(g, g.LINEAR_DX, m, n, k, g.DTYPE_BF16)
        g.grp_linear_dx(m, n, k, dz, dz.ld, w, w.ld, code(g, act), zin if act != "none" else None, zin.ld, da, da.ld, CODE[dt], ws)
        lin, size = dz.d() @ w.d().t(), dz.d().abs() @ w.d().abs().t()
        sl = slope64(zin.d(), act)
        want = lin * sl
        tol = size * (n + 12) * 2 * U * sl.abs() + (0 if act in ("none", "relu") else lin.abs() * (1 + zin.d().abs()) * 2.0 ** -20) + want.abs() * (half_step(dt) + 2 * U)
        within(da.v, want, tol * (1 + half_step(dt)))
        assert da.untouched()


@pytest.mark.parametrize("m,n,k", SHAPES + [(20001, 16, 24), (40000, 130, 70)])
def test_linear_dw(g, m, n, k):
    for pad, off, sums in [(0, 0, True), (8, 0, False), (3, 1, True)]:
        r = gen(m + n + k + pad)
        a, dz = Mat(m, k, BF16, pad, off, randn(m, k, r)), Mat(m, n, BF16, pad, off, randn(m, n, r))
        dw, db = Mat(k, n, FP32, pad, off), torch.full((n + 2,), -3.0, device=DEV)
        ws = workspace(g, g.LINEAR_DW, m, n, k, g.DTYPE_BF16)
        g.grp_linear_dw(m, n, k, a, a.ld, dz, dz.ld, dw, dw.ld, db if sums else None, ws)
        within(dw.v, a.d().t() @ dz.d(), (a.d().abs().t() @ dz.d().abs()) * (m + 12) * 2 * U)
        if sums:
            within(db[:n], dz.d().sum(0), dz.d().abs().sum(0) * (m + 12) * 2 * U)
        assert dw.untouched() and bool((db[n if sums else 0:] == -3).all())


def test_linear_gradients_against_differences(g):
    """Of a layer's loss sum(dc * act(A W + b)) in 64 bits, through dz = dc act'(z) as the kernels take it."""
    m, n, k = 9, 20, 14
    r = gen(3)
    a, w = randn(m, k, r).to(BF16), randn(k, n, r, 0.3).to(BF16)
    dz, zin = randn(m, n, r).to(BF16), randn(m, k, r).to(BF16)
    da, dw, db = torch.empty(m, k, device=DEV), torch.empty(k, n, device=DEV), torch.empty(n, device=DEV)
    g.grp_linear_dx(m, n, k, dz, n, w, n, g.ACT_GELU, zin, k, da, k, g.DTYPE_FP32, workspace(g, g.LINEAR_DX, m, n, k, 1))
    g.grp_linear_dw(m, n, k, a, k, dz, n, dw, n, db, workspace(g, g.LINEAR_DW, m, n, k, 1))

    def below(z):
        return (act64(z, "gelu") @ w.double() * dz.double()).sum()

    def layer(ww, bb):
        return ((a.double() @ ww + bb) * dz.double()).sum()

    step = 1e-5
    for i, c in [(0, 0), (8, 13), (4, 6)]:
        e = torch.zeros(m, k, device=DEV, dtype=torch.float64)
        e[i, c] = step
        assert abs(float(da[i, c]) - float(below(zin.double() + e) - below(zin.double() - e)) / (2 * step)) < 2e-5
        e = torch.zeros(k, n, device=DEV, dtype=torch.float64)
        e[c, i] = step
        zero = torch.zeros(n, device=DEV, dtype=torch.float64)
        assert abs(float(dw[c, i]) - float(layer(w.double() + e, zero) - layer(w.double() - e, zero)) / (2 * step)) < 1e-4
        e1 = torch.zeros(n, device=DEV, dtype=torch.float64)
        e1[c] = step
        assert abs(float(db[c]) - float(layer(w.double(), e1) - layer(w.double(), -e1)) / (2 * step)) < 1e-4


def test_activations_over_their_range(g):
    """Values and slopes at every size of z: the tails keep their sign and fall to zero, large ones pass."""
    z = torch.cat([torch.linspace(-40, 40, 4001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 3e38, -3e38, 88.0, -88.0, 104.0, -104.0])]).to(DEV)
    n = z.numel()
    one, a = torch.ones(1, 1, device=DEV, dtype=BF16), torch.zeros(1, 1, device=DEV, dtype=BF16)
    w = torch.zeros(1, n, device=DEV, dtype=BF16)
    for act in ACTS:
        c = torch.empty(1, n, device=DEV)
        g.grp_linear(1, n, 1, a, 1, w, n, g.DTYPE_BF16, None, None, z, code(g, act), None, 0, c, n, g.DTYPE_FP32, None, 0, workspace(g, 0, 1, n, 1, 1))
        want = act64(z.double(), act)
        within(c[0], want, (1 + z.double().abs()).clamp_max(64) * 2.0 ** -20 + want.abs() * 4 * U)
    zb = z.to(BF16)
    for act in ACTS[1:]:
        da = torch.empty(1, n, device=DEV)
        g.grp_linear_dx(1, 1, n, one, 1, torch.ones(n, 1, device=DEV, dtype=BF16), 1, code(g, act), zb, n, da, n, g.DTYPE_FP32, workspace(g, 1, 1, 1, n, 1))
        want = slope64(zb.double(), act)
        within(da[0], want, (1 + zb.double().abs()).clamp_max(64) * 2.0 ** -20)


def test_linear_infinities_stay_in_their_rows(g):
    m, n, k = 70, 200, 100
    r = gen(8)
    a, w = randn(m, k, r).to(BF16), randn(k, n, r).to(BF16)
    a[3, 5], a[69, 99] = float("inf"), float("nan")
    c = torch.empty(m, n, device=DEV)
    g.grp_linear(m, n, k, a, k, w, n, g.DTYPE_BF16, None, None, None, g.ACT_NONE, None, 0, c, n, g.DTYPE_FP32, None, 0, workspace(g, 0, m, n, k, 1))
    assert bool(c[3].isinf().all()) and bool(c[69].isnan().all())
    rest = torch.ones(m, dtype=torch.bool, device=DEV)
    rest[3] = rest[69] = False
    assert bool(c[rest].isfinite().all())


# ------------------------------------------------------------------------------------------------ clipping
@pytest.mark.parametrize("counts", [[], [0], [1], [7, 0, 9], [5000, 1, 8191, 8192, 8193, 3], [1 << 20, 12345, 2049], list(range(1, 120)), [3_000_001, 17]])
def test_clip(g, counts):
    for max_norm in (1e-2, 1e9):
        for place in ("apart", "in place"):
            r = gen(len(counts) + 1)
            ts = []
            for i, n in enumerate(counts):                                     # both types, at odd starts
                t = torch.randn(n + 3, generator=r, device=DEV).to(BF16 if i % 2 else FP32)
                ts.append(t[i % 3:i % 3 + n])
            before = [t.double() for t in ts]
            outs = None if place == "in place" else [torch.full((t.numel() + 2,), -9.0, device=DEV, dtype=t.dtype)[1:-1] for t in ts]
            norm = torch.empty(1, device=DEV)
            h = g.grp_gradients_create(ts, outs)
            g.grp_clip_gradients(h, max_norm, norm)
            want = math.sqrt(sum(float(t.square().sum()) for t in before))
            assert abs(float(norm) - want) <= want * 2 * U
            c = 1.0 if want <= max_norm else max_norm / want
            for t, b in zip(ts if outs is None else outs, before):
                within(t, b * c, b.abs() * c * (half_step(t.dtype) + 3 * U))
            if outs is not None:
                for t, b, o in zip(ts, before, outs):
                    assert torch.equal(t.double(), b)
                    assert o._base is None or bool((o._base[0] == -9) & (o._base[-1] == -9))
            h.destroy()


def test_clip_special_norms(g):
    """A norm past fp32's squares, an infinity, a NaN, and zeros."""
    for fill, want in ((1e30, 1e32), (float("inf"), float("inf")), (float("nan"), float("nan")), (0.0, 0.0)):
        t = torch.full((10_000,), fill, device=DEV)
        norm = torch.empty(1, device=DEV)
        h = g.grp_gradients_create([t])
        g.grp_clip_gradients(h, 1.0, norm)
        assert float(norm) == pytest.approx(want, rel=1e-6, nan_ok=True)
        if fill == 1e30:
            within(t, torch.full_like(t, 1e-2).double(), 1e-2 * 4 * U)
        elif fill == 0.0:
            assert bool((t == 0).all())
        else:
            assert bool(t.isnan().all())             # inf * 0, and NaN, as the formula has it


# ------------------------------------------------------------------------------------------------ streams, graphs, repeats
def block_pass(g, s):
    """One forward and backward pass of a residual block and the clipping of its gradient, on the current stream."""
    m, d, f = s["m"], s["d"], s["f"]
    g.grp_rmsnorm(m, d, s["x"], d, g.DTYPE_BF16, s["r"], d, s["w"], 1e-6, s["h"], d, s["y"], d, g.DTYPE_BF16)
    g.grp_linear(m, f, d, s["y"], d, s["w1"], f, g.DTYPE_BF16, None, None, s["b1"], g.ACT_GELU, None, 0, s["a"], f, g.DTYPE_BF16, s["z"], f, s["ws"])
    g.grp_linear(m, d, f, s["a"], f, s["w2"], d, g.DTYPE_BF16, None, None, None, g.ACT_NONE, s["h"], d, s["out"], d, g.DTYPE_BF16, None, 0, s["ws"])
    g.grp_linear_dx(m, d, f, s["dout"], d, s["w2"], d, g.ACT_GELU, s["z"], f, s["dz"], f, g.DTYPE_BF16, s["ws"])
    g.grp_linear_dw(m, d, f, s["a"], f, s["dout"], d, s["dw2"], d, s["db2"], s["ws"])
    g.grp_linear_dx(m, f, d, s["dz"], f, s["w1"], f, g.ACT_NONE, None, 0, s["dy"], d, g.DTYPE_BF16, s["ws"])
    g.grp_linear_dw(m, f, d, s["y"], d, s["dz"], f, s["dw1"], f, s["db1"], s["ws"])
    g.grp_rmsnorm_backward(m, d, s["dy"], d, g.DTYPE_BF16, s["h"], d, g.DTYPE_BF16, s["w"], 1e-6, s["dout"], d, s["dh"], d, s["dw"], s["ws"])
    g.grp_clip_gradients(s["handle"], 1e-3, s["norm"])


OUTS = ("h", "y", "a", "z", "out", "dz", "dw2", "db2", "dy", "dw1", "db1", "dh", "dw", "norm")


def block_state(g, m=700, d=96, f=200):
    r = gen(4)
    s = {"m": m, "d": d, "f": f}
    for name, shape in (("x", (m, d)), ("r", (m, d)), ("dout", (m, d)), ("w1", (d, f)), ("w2", (f, d))):
        s[name] = (torch.randn(*shape, generator=r, device=DEV) * (0.1 if name[0] == "w" else 1.0)).to(BF16)
    s["w"], s["b1"] = 1 + 0.1 * torch.randn(d, generator=r, device=DEV), torch.randn(f, generator=r, device=DEV)
    for name, shape in (("h", (m, d)), ("y", (m, d)), ("a", (m, f)), ("z", (m, f)), ("out", (m, d)), ("dz", (m, f)), ("dy", (m, d)), ("dh", (m, d))):
        s[name] = torch.empty(*shape, device=DEV, dtype=BF16)
    for name, shape in (("dw1", (d, f)), ("dw2", (f, d)), ("db1", (f,)), ("db2", (d,)), ("dw", (d,)), ("norm", (1,))):
        s[name] = torch.empty(*shape, device=DEV)
    need = [g.grp_linear_workspace_bytes(kind, m, n, k, g.DTYPE_BF16) for kind in (0, 1, 2) for n, k in ((d, f), (f, d))]
    s["ws"] = torch.empty(max(need + [g.grp_rmsnorm_backward_workspace_bytes(m, d), 1]), dtype=torch.uint8, device=DEV)
    s["handle"] = g.grp_gradients_create([s[k] for k in ("dw1", "dw2", "db1", "db2", "dw")])
    return s


def test_equal_inputs_give_equal_bits_on_every_stream_and_in_graphs(g):
    s = block_state(g)
    block_pass(g, s)
    torch.cuda.synchronize()
    want = {k: s[k].clone() for k in OUTS}
    assert all(bool(v.float().isfinite().all()) for v in want.values())

    def check():
        torch.cuda.synchronize()
        for k in OUTS:
            assert torch.equal(s[k], want[k]), k
            s[k].zero_()
        torch.cuda.synchronize()

    check()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        block_pass(g, s)
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        block_pass(g, s)
    for _ in range(3):
        graph.replay()
        check()
        block_pass(g, s)
        check()


# ------------------------------------------------------------------------------------------------ large
def test_offsets_past_32_bits(g):
    """Rows that begin beyond 2^31 elements (and 2^32 bytes): the last ones, and those around the border."""
    m, k, n = 140_001, 16_384, 16
    r = gen(1)
    a = torch.empty(m, k, device=DEV, dtype=BF16)
    for i in range(0, m, 20_000):
        a[i:i + 20_000] = torch.randn(min(20_000, m - i), k, generator=r, device=DEV)
    rows = [0, 65_535, 65_536, 131_071, 131_072, 131_073, m - 1]
    x = a[rows].double()
    y = torch.empty_like(a)
    g.grp_rmsnorm(m, k, a, k, g.DTYPE_BF16, None, 0, None, 1e-6, None, 0, y, k, g.DTYPE_BF16)
    want = x / torch.sqrt(x.square().mean(1, keepdim=True) + 1e-6)
    within(y[rows], want, want.abs() * (half_step(BF16) + 80 * U))
    ws = torch.empty(g.grp_rmsnorm_backward_workspace_bytes(m, k), dtype=torch.uint8, device=DEV)
    dw = torch.empty(k, device=DEV)
    g.grp_rmsnorm_backward(m, k, a, k, g.DTYPE_BF16, a, k, g.DTYPE_BF16, None, 1e-6, None, 0, y, k, dw, ws)
    dh, size, _, _ = norm_grad64(x, x, 1.0, 1e-6, 0.0)
    within(y[rows], dh, dh.abs() * half_step(BF16) + size * 160 * U)
    w = torch.randn(k, n, generator=r, device=DEV).to(BF16)
    c = torch.empty(m, n, device=DEV)
    g.grp_linear(m, n, k, a, k, w, n, g.DTYPE_BF16, None, None, None, g.ACT_NONE, None, 0, c, n, g.DTYPE_FP32, None, 0, workspace(g, 0, m, n, k, 1))
    within(c[rows], x @ w.double(), (x.abs() @ w.double().abs()) * (k + 12) * 2 * U)
    dz = torch.randn(m, n, generator=r, device=DEV).to(BF16)
    dwt = torch.empty(k, n, device=DEV)
    g.grp_linear_dw(m, n, k, a, k, dz, n, dwt, n, None, workspace(g, 2, m, n, k, 1))
    for at in (slice(0, 32), slice(k - 32, k)):
        p = a[:, at].double()
        within(dwt[at], p.t() @ dz.double(), (p.abs().t() @ dz.double().abs()) * (m + 12) * 2 * U)
    da = y
    g.grp_linear_dx(m, n, k, dz, n, w, n, g.ACT_RELU, a, k, da, k, g.DTYPE_BF16, workspace(g, 1, m, n, k, 1))
    lin = dz[rows].double() @ w.double().t()
    within(da[rows], lin * (x > 0), (dz[rows].double().abs() @ w.double().abs().t()) * (n + 12) * 2 * U + lin.abs() * half_step(BF16) * 1.01)
