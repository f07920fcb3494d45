"""8-bit products with large ones among them that cancel: what the header promises of sums in fp32 (C of fp32) and of the 8-bit instructions' (C of bf16)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4M3, BF16, FP32 = torch.float8_e4m3fn, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def g():
    import paper_2602_01872_amd as lib
    lib.load()
    return lib


@pytest.mark.parametrize("m,n,k", [(1, 32, 16), (20, 40, 24), (64, 300, 128), (300, 136, 272), (300, 137, 271), (1000, 520, 128)])
@pytest.mark.parametrize("apart", [1, 3, 9])
def test_outliers_that_cancel(g, m, n, k, apart):
    """Two of A's columns hold 448 and meet 448 and -448: of a result of at most k the products have sizes of 2 x 200704.  fp32 sums are off by (k + 12) 2^-23 of
    those, the 8-bit instructions by 7 2^-13, which is stated, and z as C."""
    r = torch.Generator(device=DEV)
    r.manual_seed(m + k)
    a = torch.randint(-1, 2, (m, k), generator=r, device=DEV).float()
    w = torch.randint(-1, 2, (n, k), generator=r, device=DEV).float()
    at = torch.randint(0, k - apart, (n,), generator=r, device=DEV)[0]
    a[:, at], a[:, at + apart] = 448, 448
    w[:, at], w[:, at + apart] = 448, -448
    lin, size = a.double() @ w.double().t(), a.double().abs() @ w.double().abs().t()
    aq, wq = a.to(E4M3), w.to(E4M3)
    assert torch.equal(aq.float(), a) and torch.equal(wq.float(), w)
    for ct, part in ((FP32, (k + 12) * 2.0 ** -23), (BF16, 7 * 2.0 ** -13)):
        c, z = torch.empty(m, n, device=DEV, dtype=ct), torch.empty(m, n, device=DEV, dtype=BF16)
        b = g.grp_linear_workspace_bytes(g.LINEAR_FORWARD, m, n, k, g.DTYPE_E4M3)
        g.grp_linear(m, n, k, aq, k, wq, k, g.DTYPE_E4M3, None, None, None, g.ACT_NONE, None, 0, c, n, g.DTYPE_FP32 if ct is FP32 else g.DTYPE_BF16, z, n,
                     torch.empty(b, dtype=torch.uint8, device=DEV) if b else None)
        for got, t in ((c, ct), (z, BF16)):
            half = torch.finfo(t).eps / 2
            assert bool(((got.double() - lin).abs() <= size * part * (1 + half) + lin.abs() * half).all())
